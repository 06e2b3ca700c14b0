// Attention of new tokens over a list of the paged 8-bit cache that several sequences
// share, and over each sequence's own list.
//
// softmax over both lists together: each is cut into pieces as in the plain
// attention, every piece gives (O, m, l) of its rows, and the pieces of both are joined,
//   O = sum 2^(m_x - m) O_x / sum 2^(m_x - m) l_x,   m = max m_x.
// A piece of the shared list serves the rows of all sequences that share it, so the list is read
// once for tiles of 16, 32 or 128 of them and not once a sequence.  Each wave decodes what it
// reads: a page once for a tile of 16 or 32 rows, whose waves take pages in turn, and four times
// for 128, whose waves take 32 rows of the same page each.  Both lists' pieces are workgroups of
// one launch, the shared ones first: they are bound by instructions where there are many rows and
// the own lists' by memory.
//
// One token of each of 32 samples over 35,840 shared and up to 2,048 own tokens, 40/8 heads of 128:
// 59 to 64 us with the card's clock; the plain attention over tables that all name the shared pages
// takes 159 where this takes 64.  Two samples' frames of 1,792 tokens over 35,840 and 3,584, 12
// heads: 927 to 968 us, 0.9 PFLOP/s, the plain attention so 926 where this takes 967: their rows
// fill the tiles either way, and the partial results' way to memory is not needed there.  Tried: a
// tile's walk over the shared list and then its own as one list (frames 954 us), the next page's
// keys requested during a page's softmax, into the registers that its scores leave free (59.2 and
// 59.4 us; D = 64 18.2 and 19.1).
#include <algorithm>

#include "cache_tile.hpp"

namespace vsa2 {

namespace {

// How the two sides are cut.
struct side_plan {
    int tile_rows;
    int64_t tiles;
    int splits;
    int64_t lists;
    int64_t items() const { return lists * tiles; }
    // a multiple of eight, so that both sides' pieces start at the same XCD
    int64_t blocks(bool spread) const {
        const int64_t pieces = lists * splits;
        return ((spread ? (pieces + 7) / 8 * 8 : pieces) * tiles + 7) / 8 * 8;
    }
    size_t floats(int D) const { return static_cast<size_t>(items()) * splits * tile_rows * (D + 2); }
};
struct shared_plan {
    side_plan pre, own;
};

// A body for the shared rows and one for the own rows: tiles of 16 X rows, or 0 for 128.
template <int D, int X> struct lds_of { using type = tile_lds<D, 4, X>; };
template <int D> struct lds_of<D, 0> { using type = rows_lds<D>; };

template <typename T, int D, int X, rows_kind KIND>
__device__ __forceinline__ void side_body(const attn_args& a, uint32_t block, uint32_t blocks, char* lds) {
    auto& mine = *reinterpret_cast<typename lds_of<D, X>::type*>(lds);
    if constexpr (X == 0) rows_body<T, D, KIND>(a, plain_scores{}, block, blocks, mine);
    else tile_body<T, D, 4, X, KIND>(a, plain_scores{}, block, blocks, mine);
}

template <typename T, int D, int PRE, int OWNX>
__global__ __launch_bounds__(256, sizeof(T) == 4 && D == 128 && PRE == 0 ? 1 : 2) void attn_shared_kernel(
    attn_args pre, attn_args own, uint32_t pre_blocks) {
    constexpr size_t A = sizeof(typename lds_of<D, PRE>::type), B = sizeof(typename lds_of<D, OWNX>::type);
    __shared__ __attribute__((aligned(1024))) char lds[A > B ? A : B];
    if (blockIdx.x < pre_blocks) side_body<T, D, PRE, SHARED>(pre, blockIdx.x, pre_blocks, lds);
    else side_body<T, D, OWNX, OWN>(own, blockIdx.x - pre_blocks, gridDim.x - pre_blocks, lds);
}

// Joins a row's pieces of both lists, the shared one's first, as attn_cache_join_kernel does.
template <typename T, int D, int SLICES>
__global__ __launch_bounds__(SLICES > 8 ? 32 * SLICES : 256) void shared_join_kernel(attn_args pre, attn_args own, int pre_tile,
                                                                                     int own_tile) {
    constexpr int RPW = SLICES > 8 ? 1 : 8 / SLICES;       // rows of a workgroup
    __shared__ float so[SLICES > 1 ? SLICES : 1][D], sl[SLICES];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, slice = group % SLICES;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * RPW + group / SLICES;
    const int64_t bh = at / own.rows;
    if (bh >= static_cast<int64_t>(own.c.batch) * own.c.heads) return;      // all lanes of a row together
    const int rr = static_cast<int>(at - bh * own.rows);
    const int b = static_cast<int>(bh / own.c.heads), h = static_cast<int>(bh % own.c.heads);
    // a row's pieces on either side: where its elements and its (m, l) start, and the pieces' stride
    struct pieces {
        const float *o, *ml;
        int64_t stride;
    };
    const auto pieces_of = [](const attn_args& a, int64_t list, int row, int tile_rows) {
        const int64_t stride = static_cast<int64_t>(tile_rows) * (D + 2);
        const int tile = row / tile_rows, in = row - tile * tile_rows;
        const float* p = a.part + (list * a.tiles + tile) * a.splits * stride;
        return pieces{p + in * D, p + static_cast<int64_t>(tile_rows) * D + 2 * in, stride};
    };
    const pieces far = pieces_of(pre, static_cast<int64_t>(b / pre.samples) * pre.c.heads + h,
                                 b % pre.samples * own.rows + rr, pre_tile);
    const pieces near = pieces_of(own, bh, rr, own_tile);
    const int first = pre.splits, all = pre.splits + own.splits;
    const auto ml_of = [&](int x) {
        return *reinterpret_cast<const float2*>(x < first ? far.ml + x * far.stride : near.ml + (x - first) * near.stride);
    };
    float m = -INFINITY;
    for (int x = lane; x < all; x += 32) m = fmaxf(m, ml_of(x).x);
#pragma unroll
    for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k, 64));
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f, o[D / 32] = {};
    // 32 of this slice's pieces at a time: their weights one a lane, then their sums
    for (int x0 = slice; x0 < all; x0 += 32 * SLICES) {
        float f = 0.f;
        if (x0 + lane * SLICES < all) {
            const float2 y = ml_of(x0 + lane * SLICES);
            f = fast_exp2(y.x - base);
            l += f * y.y;
        }
        const int n = min(32, (all - x0 + SLICES - 1) / SLICES);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const int x = x0 + i * SLICES;
            const float* px = (x < first ? far.o + x * far.stride : near.o + (x - first) * near.stride) + lane * (D / 32);
            const float w = __shfl(f, (threadIdx.x & 32) + i, 64);
#pragma unroll
            for (int k = 0; k < D / 32; ++k) o[k] += w * px[k];
        }
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) l += __shfl_xor(l, k, 64);
    if constexpr (SLICES > 1) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) so[slice][lane * (D / 32) + i] = o[i];
        if (lane == 0) sl[slice] = l;
        __syncthreads();
        if (slice) return;
#pragma unroll
        for (int x = 1; x < SLICES; ++x) {
            l += sl[x];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) o[i] += so[x][lane * (D / 32) + i];
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = static_cast<T*>(own.o.ptr) + row_offset(own.o, own, b, h, rr) + lane * (D / 32);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) from_f32(out[i], l == 0.f ? 0.f : o[i] * inv);
    if (lane == 0) store_lse(own, b, h, rr, base, l);
}

// What a workgroup's piece of `pages` takes, in us: a start and an end, then its pages, which
// tiles' waves share out and rows' waves walk together.  Measured with two workgroups a CU (one
// alone is faster by a third): 35,840 shared tokens, 8 heads of 128, 160 rows in pieces for 160
// to 1,000 workgroups 45 to 67 us, this with 18 us around it within 4 of them.  A page of D = 64, or of
// fp32 rows, takes other times, but all pieces' alike: of 56 pairs of numbers of pieces from 2 to 256 and
// 1 to 8 the rule's was within 1% of the fastest in seven calls (32 tokens over 35,840, D = 64: bf16 41.6 us,
// best 41.8, fp32 56.1 and 55.5, fp32 of D = 128 89.4 and 91.1; D = 64, 2 x 8 tokens over 20,000 18.3 and
// 18.2, 4 x 16 over 8,000 21.1 and 21.2, 600 rows over 20,000 63.3 and 62.9; fp32, 64 over 17,000 27.4 and 27.4).
double piece_time(const side_plan& p, int dtype, int64_t pages, bool pairs) {
    const int64_t n = (pages + p.splits - 1) / p.splits;
    const double page = p.tile_rows == ROWS ? 2.4 : (pairs ? 2. : 1.5);
    return 3. + (p.tile_rows == ROWS ? n : (n + 3) / 4) * (dtype == 0 ? 2. * page : page);
}

// Both sides' pieces on the 512 slots of two workgroups a CU, the shared ones first: when the last one
// ends, and the partial results' way to memory and back.
double call_time(const shared_plan& p, int dtype, int D, const int64_t (&pages)[2], const int64_t (&rows)[2], bool pairs) {
    constexpr double SLOTS = 512.;
    const double pre = piece_time(p.pre, dtype, pages[0], pairs), own = piece_time(p.own, dtype, pages[1], false);
    const double n = static_cast<double>(p.pre.items()) * p.pre.splits;
    double left = static_cast<double>(p.own.items()) * p.own.splits;
    // slots by when they are free: `later` of them a piece after the others
    const double rounds = static_cast<double>(static_cast<int64_t>(n / SLOTS)), later = n - rounds * SLOTS;
    double early = rounds * pre, late = later > 0 ? early + pre : early;
    const double step = left > 8 * SLOTS ? static_cast<double>(static_cast<int64_t>(left / SLOTS / 4)) : 1.;
    while (left > 0) {
        if (early <= late || later == 0) {
            left -= (SLOTS - later) * step;
            early += own * step;
        } else {
            left -= later * step;
            late += own * step;
        }
    }
    const double bytes = 8. * (D + 2) * rows[1] * p.own.lists * (p.pre.splits + p.own.splits);
    return std::max(early, later > 0 ? late : early) + bytes / 4e6;
}

shared_plan plan_shared(int dtype, int D, const cache_view& pre, const cache_view& c, int heads_q, int n) {
    shared_plan p;
    const int64_t own_rows = static_cast<int64_t>(heads_q / c.heads) * n, pre_rows = own_rows * (c.batch / pre.batch);
    const bool pairs = !(dtype == 0 && D == 128);
    p.own.lists = static_cast<int64_t>(c.batch) * c.heads;
    p.pre.lists = static_cast<int64_t>(pre.batch) * c.heads;
    // Shared rows in tiles of 32 up to 512 of them, else of 128, whose waves share the pages.  35,840
    // shared tokens, 8 heads of 128, up to 512 own ones (us, tiles of 32 against 128): 130 rows 50
    // and 69, 200 68 and 64, 240 76 and 85, 320 85 and 91, 640 147 and 138.
    p.own.tile_rows = own_rows <= 64 ? TILE : ROWS;
    p.pre.tile_rows = own_rows > 64 || pre_rows > 512 ? ROWS : (pairs ? 2 * TILE : TILE);
    const int64_t rows[2] = {pre_rows, own_rows}, pages[2] = {pre.max_pages, c.max_pages};
    side_plan* side[2] = {&p.pre, &p.own};
    int64_t most[2];
    for (int x = 0; x < 2; ++x) {
        side[x]->tiles = (rows[x] + side[x]->tile_rows - 1) / side[x]->tile_rows;
        side[x]->splits = 1;
        const int per = side[x]->tile_rows == ROWS ? 8 : 4;          // pages a piece has at least
        most[x] = std::max<int64_t>(1, std::min<int64_t>((pages[x] + per - 1) / per, 1024 / side[x]->items()));
    }
    // the shared list for whole and half rounds of the slots, with and beside the own pieces
    shared_plan best = p;
    double least = -1.;
    for (int64_t s = 1; s <= most[1]; s *= 2) {
        for (int half = 1; half <= 4; ++half)
            for (int beside = 0; beside < 2; ++beside) {
                const int64_t room = 256 * half - beside * p.own.items() * s;
                p.own.splits = static_cast<int>(s);
                p.pre.splits = static_cast<int>(std::max<int64_t>(1, std::min(most[0], room / p.pre.items())));
                const double t = call_time(p, dtype, D, pages, rows, pairs);
                if (least < 0. || t < least) {
                    least = t;
                    best = p;
                }
            }
    }
    return best;
}

// The pieces of either side spread over the XCDs as plan_args has it.
bool spreads(const side_plan& p) { return p.tile_rows != ROWS || p.lists * p.splits >= 128; }

template <typename T, int D, int PRE, int OWNX>
void launch_pieces(const attn_args& pre, const attn_args& own, const shared_plan& p, hipStream_t s) {
    const uint32_t first = static_cast<uint32_t>(p.pre.blocks(pre.spread));
    const dim3 grid(first + static_cast<uint32_t>(p.own.blocks(own.spread)));
    hipLaunchKernelGGL((attn_shared_kernel<T, D, PRE, OWNX>), grid, dim3(256), 0, s, pre, own, first);
}

template <typename T, int D>
void launch_shared(const attn_args& pre, const attn_args& own, const shared_plan& p, hipStream_t s) {
    if (p.own.tile_rows == ROWS) launch_pieces<T, D, 0, 0>(pre, own, p, s);
    else if (p.pre.tile_rows == ROWS) launch_pieces<T, D, 0, 1>(pre, own, p, s);
    else launch_pieces<T, D, two_tiles<T, D> ? 2 : 1, 1>(pre, own, p, s);
    const int64_t rows = static_cast<int64_t>(own.c.batch) * own.c.heads * own.rows;
    const int pieces = p.pre.splits + p.own.splits, pt = p.pre.tile_rows, ot = p.own.tile_rows;
    const auto groups = [&](int per_wg) { return dim3(static_cast<unsigned>((rows + per_wg - 1) / per_wg)); };
    if (pieces > 32)
        hipLaunchKernelGGL((shared_join_kernel<T, D, 32>), groups(1), dim3(1024), 0, s, pre, own, pt, ot);
    else if (pieces > 8)
        hipLaunchKernelGGL((shared_join_kernel<T, D, 8>), groups(1), dim3(256), 0, s, pre, own, pt, ot);
    else
        hipLaunchKernelGGL((shared_join_kernel<T, D, 1>), groups(8), dim3(256), 0, s, pre, own, pt, ot);
}

}  // namespace

size_t attn_cache_shared_workspace_bytes(const cache_view& pre, const cache_view& c, int D, int heads_q, int n) {
    size_t most = 0;
    for (int dtype = 0; dtype < 2; ++dtype) {
        const shared_plan p = plan_shared(dtype, D, pre, c, heads_q, n);
        most = std::max(most, (p.pre.floats(D) + p.own.floats(D)) * sizeof(float));
    }
    return most;
}

hipError_t launch_attn_cache_shared(int dtype, int D, const cache_view& pre, const cache_view& c, int heads_q, int n,
                                    const row_view& q, const int32_t* pre_length, const int32_t* length,
                                    const int32_t* count, bool causal, const row_view& o, float* lse, void* ws,
                                    hipStream_t s) {
    const shared_plan p = plan_shared(dtype, D, pre, c, heads_q, n);
    const auto args = [&](const side_plan& y, const cache_view& v, const int32_t* len, float* part, int samples) {
        attn_args a = plan_args(attn_plan{y.tile_rows, 4, y.tiles, y.splits}, v, heads_q, n, q, len, count, causal, o, lse, part);
        a.samples = samples;
        a.rows *= samples;
        a.spread = spreads(y);
        return a;
    };
    const attn_args far = args(p.pre, pre, pre_length, static_cast<float*>(ws), c.batch / pre.batch);
    const attn_args own = args(p.own, c, length, static_cast<float*>(ws) + p.pre.floats(D), 1);
    if (dtype == 0 && D == 64) launch_shared<float, 64>(far, own, p, s);
    else if (dtype == 0) launch_shared<float, 128>(far, own, p, s);
    else if (D == 64) launch_shared<bf16_t, 64>(far, own, p, s);
    else launch_shared<bf16_t, 128>(far, own, p, s);
    return hipGetLastError();
}

}  // namespace vsa2
