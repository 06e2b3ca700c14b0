// Attention of new tokens over the paged 8-bit cache.
//
// Rows: the query heads of one KV head times the call's tokens (token-major), in
// tiles of 16 (or pairs of them, or 128).  Everything is computed transposed, S^T = K Q^T and
// O^T = V^T P^T on 16x16x32 MFMAs, so that a lane holds one row (column
// lane % 16) through the whole kernel: the softmax needs two exchanges a page,
// P goes from the accumulators of the first product into the operand of the
// second without leaving its lane (the page's V order is made for that), and O
// is rescaled lane by lane.  e4m3 codes become 16-bit values exactly: K's bf16,
// with the token's power applied by the conversion, V's plain, with the power
// on P.  fp32 queries and probabilities are three bf16 terms each, so their
// products lose nothing that fp32 sums would keep.  For bf16 queries P and V
// are fp16: 11 bits of a weight, where bf16's 8 would cost as much as the
// result's own rounding.  fp16's exponents do not reach far: P is scaled by a
// power of two that makes the largest power seen 2^7, and in rows whose weight is
// on tokens of much smaller powers by one more (row_softmax).  Measured against
// bf16 P: 3% of the time at 1,792 rows, 3 to 9% over a few rows where codes and
// weights bound a page (D = 64), none where memory does; where every page holds
// powers 2^7 apart or more, 17 to 26% there.
//
// Bound by memory for single tokens: 2 (D + 1) bytes per token and KV head.  A
// page is 16 KB in runs of 1 KB per load instruction; the waves of a workgroup
// and the workgroups of a split take different pages of a list, each with its
// own running maximum and sum, and are joined at the end in a fixed order.  16
// sequences of 20,000 to 76,800 tokens, 40 query and 8 KV heads of 128: 281 us, 5.7
// TB/s.  For many rows bound by vector instructions, which hardly overlap with the
// MFMAs of two waves a SIMD: 1,792 tokens over 35,840, 12 heads, 430 us, 0.92
// PFLOP/s; vector unit busy 63% of the cycles and MFMAs 43%, waits for LDS 1%.
//
// The waves' code is in cache_tile.hpp; this file holds the kernels around it and the rules
// by which a call is cut.
#include <algorithm>

#include "cache_tile.hpp"

namespace vsa2 {

namespace {

template <typename T, int D, int WAVES, int XT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, D == 128 ? 2 : 4))) void attn_cache_kernel(
    attn_args a) {
    __shared__ tile_lds<D, WAVES, XT> lds;
    tile_body<T, D, WAVES, XT, WHOLE>(a, plain_scores{}, blockIdx.x, gridDim.x, lds);
}
template <typename T, int D>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 4 ? 1 : 2) void attn_cache_rows_kernel(attn_args a) {
    __shared__ rows_lds<D> lds;
    rows_body<T, D, WHOLE>(a, plain_scores{}, blockIdx.x, gridDim.x, lds);
}

// Which kernel: tiles of 16 or 32 rows whose waves share out a list's pages, or
// 128-row tiles whose waves share the pages.  The first reads and decodes a page
// once per tile but splits finely; measured over lists of 20,000 tokens (us,
// tiles of 16 and of 32 against 128-row ones): bf16, D = 128, 8 lists of 128 rows
// 33 and 31 against 42, 32 of 96 rows 68 and 55 against 65, of 128 rows 94 and 72
// against 72, 128 lists of 64 rows 193 and 154 against 196, of 96 rows 264 and 201
// against 204; fp32, D = 128, 32 lists of 128 rows 131 against 127.  fp32 at D = 64
// would gain from pairs also at 128 lists of 96 rows (lists of uneven lengths 151 and
// 138 against 170), which the limit of 64 lists, drawn for D = 128, leaves out.
bool takes_tiles(int dtype, int D, int64_t lists, int64_t rows) {
    return rows <= 64 || (rows <= 128 && ((dtype == 0 && D == 128) || lists < 64));
}

// Small tiles of 32 rows: half the decoding, where there are workgroups enough
// either way.  Measured with 128 lists (us, 16 rows against 32): lists of 40,000
// tokens, bf16, D = 128, 32 / 48 / 64 rows 248 / 325 / 366 against 250 / 271 / 280;
// D = 64 140 / 173 / 212 against 135 / 183 / 187 (a half-empty pair costs more than
// it saves there); 5,000 tokens 35 / 44 / 44 against 36 / 42 / 42.  Of short
// lists, where a pair makes the tiles one and the call one launch: 32 rows of 1,000
// tokens 16.3 against 15.0.
bool takes_pairs(int dtype, int D, int64_t lists, int64_t rows, int pages) {
    const int64_t tiles = (rows + TILE - 1) / TILE;
    if (tiles == 1 || (dtype == 0 && D == 128) || lists * tiles < 128) return false;
    if (pages <= 32) return tiles == 2;
    return pages >= 128 && (tiles % 2 == 0 || (dtype == 1 && D == 128));
}

}  // namespace

attn_plan plan_attn(int dtype, int D, const cache_view& c, int heads_q, int n) {
    attn_plan p;
    const int64_t rows = static_cast<int64_t>(heads_q / c.heads) * n, lists = static_cast<int64_t>(c.batch) * c.heads;
    if (takes_tiles(dtype, D, lists, rows)) {
        p.tile_rows = takes_pairs(dtype, D, lists, rows, c.max_pages) ? 2 * TILE : TILE;
        p.tiles = (rows + p.tile_rows - 1) / p.tile_rows;
        // A list in one piece takes eight waves that join it without a second
        // launch: short ones, and those of many sequences up to 200 pages.  One
        // token, in one piece against several (us): 12 lists of 1,792 tokens, bf16
        // 10.9 against 11.1, fp32 (D = 128) 14.0 against 11.3; 128 lists of 4,000,
        // bf16 24.8 against 28.5 (uneven lengths 21.0 against 23.3), fp32 29.0
        // against 30.2 (28.1 against 24.5); 192 of 6,000, bf16 48 against 56 (36
        // against 37), fp32 50 against 59 (41 against 41).  Near 200 pages uneven
        // lengths lose: 128 of up to 12,000, bf16, D = 128 79 against 78, uneven 55
        // against 48, D = 64 37 against 38 and 36 against 29; 192, fp32, D = 64 52
        // against 44.
        const int one = lists >= (dtype == 1 ? 128 : 192) ? 200 : (dtype == 0 && D == 128 && lists < 128 ? 16 : 32);
        if (p.tiles == 1 && c.max_pages <= one) {
            p.waves = 8;
            p.splits = 1;
            return p;
        }
        // Else the 512 workgroups of four waves that are resident at once (D = 128),
        // and a page for every wave at least; 256 where the pieces of few rows take
        // longer to join than they save (one token over 200,000: 512 workgroups 29
        // us, 256 23); 1,024 from 128 lists on, where the lengths, which only the GPU
        // knows, may be uneven and the pieces stay long.  One token over up to 40,000,
        // D = 128, 512 workgroups against 1,024 (us; even, uneven lengths): 96 lists
        // 176, 122 against 187, 121; 112 205, 142 against 206, 137; 128 232, 159
        // against 232, 155; 160 285, 193 against 287, 189; 256 443, 298 against 450,
        // 289; D = 64, 96 lists 94, 63 against 102, 60, 128 119, 88 against 125, 86.
        // 16 x 8 lists of 20,000 to 76,800: 299 against 287, 2,048 287.
        p.waves = 4;
        const int64_t items = lists * p.tiles, most = (c.max_pages + 3) / 4, pages64 = c.max_pages / 64;
        int64_t want = (dtype == 1 && p.tiles == 1 && items <= 16 ? 256 : 512) / items;
        if (items >= 128) want = std::max(want, std::min(1024 / items, pages64));
        p.splits = static_cast<int>(std::max<int64_t>(1, std::min(want, most)));
        return p;
    }
    p.tile_rows = ROWS;
    p.waves = NW;
    p.tiles = (rows + ROWS - 1) / ROWS;
    // Rounds of the resident workgroups (two a CU; one for fp32 at D = 128), against
    // the one that evenly spread work would take; a split adds the partial results'
    // way to memory and back, which measured 1% of a list of 36,000 tokens.
    const int64_t resident = dtype == 0 && D == 128 ? 256 : 512;
    const int64_t items = lists * p.tiles, most = (c.max_pages + 7) / 8;
    double best = 0.;
    p.splits = 1;
    for (int64_t k = 1; k <= most && (k == 1 || items * k <= 8 * resident); ++k) {
        const int64_t rounds = (items * k + resident - 1) / resident;
        const double cost = static_cast<double>(rounds) / k +
                            (k > 1 ? k * 360. / (64. * c.max_pages) * items / resident : 0.);
        if (k == 1 || cost < best) {
            best = cost;
            p.splits = static_cast<int>(k);
        }
    }
    return p;
}

size_t attn_cache_workspace_bytes(const cache_view& c, int D, int heads_q, int n) {
    size_t most = 0;
    for (int dtype = 0; dtype < 2; ++dtype) {
        const attn_plan p = plan_attn(dtype, D, c, heads_q, n);
        const size_t need = p.splits == 1 ? 0 : static_cast<size_t>(c.batch) * c.heads * p.tiles * p.splits *
                                                    p.tile_rows * (D + 2) * sizeof(float);
        if (need > most) most = need;
    }
    return most;
}

attn_args plan_args(const attn_plan& p, const cache_view& c, int heads_q, int n, const row_view& q, const int32_t* length,
                    const int32_t* count, bool causal, const row_view& o, float* lse, void* ws) {
    attn_args a{};
    a.c = c;
    a.q = q;
    a.o = o;
    a.lse = lse;
    a.length = length;
    a.count = count;
    a.part = static_cast<float*>(ws);
    a.n = n;
    a.group = heads_q / c.heads;
    a.rows = a.group * n;
    a.tiles = static_cast<int>(p.tiles);
    a.splits = p.splits;
    a.samples = 1;
    a.causal = causal;
    a.pieces = static_cast<uint32_t>(static_cast<int64_t>(c.batch) * c.heads * p.splits);
    a.spread = p.tile_rows != ROWS || a.pieces >= 128;
    return a;
}

namespace {

struct plain_kernels {
    template <typename T, int D, int WAVES, int XT>
    void tiles(dim3 grid, dim3 block, hipStream_t s, const attn_args& a) const {
        hipLaunchKernelGGL((attn_cache_kernel<T, D, WAVES, XT>), grid, block, 0, s, a);
    }
    template <typename T, int D>
    void rows(dim3 grid, dim3 block, hipStream_t s, const attn_args& a) const {
        hipLaunchKernelGGL((attn_cache_rows_kernel<T, D>), grid, block, 0, s, a);
    }
};

}  // namespace

hipError_t launch_attn_cache(int dtype, int D, const cache_view& c, int heads_q, int n, const row_view& q,
                             const int32_t* length, const int32_t* count, bool causal, const row_view& o, float* lse,
                             void* ws, hipStream_t s) {
    const attn_plan p = plan_attn(dtype, D, c, heads_q, n);
    const attn_args a = plan_args(p, c, heads_q, n, q, length, count, causal, o, lse, ws);
    const plain_kernels go;
    if (dtype == 0 && D == 64) launch_attn<float, 64>(a, p, s, go);
    else if (dtype == 0) launch_attn<float, 128>(a, p, s, go);
    else if (D == 64) launch_attn<bf16_t, 64>(a, p, s, go);
    else launch_attn<bf16_t, 128>(a, p, s, go);
    return hipGetLastError();
}

}  // namespace vsa2
