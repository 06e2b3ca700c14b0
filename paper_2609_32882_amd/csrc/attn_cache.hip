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
#include <algorithm>
#include <cfloat>

#include "common.hpp"

namespace vsa2 {

namespace {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;

constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.44269504088896340f;
constexpr int TILE = 16;          // rows of a tile of attn_cache_kernel
constexpr int NW = 4;             // waves of a workgroup of attn_cache_rows_kernel
constexpr int ROWS = 32 * NW;     // its rows
constexpr int STAGE = 2;          // pages it copies at a time

struct attn_args {
    cache_view c;
    row_view q, o;
    float* lse;
    const int32_t* length;
    const int32_t* count;
    float* part;         // [items][splits]: O [tile rows][D], then (m, l) [tile rows][2] of each
    int n, group, rows, tiles, splits;
    uint32_t pieces;     // of all lists
    bool causal, spread;
};

template <typename T> constexpr int terms_of = sizeof(T) == 4 ? 3 : 1;

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_vt;
struct frag_f16 { f16x8_t v; };

// P and V: fp16 for bf16 queries, three bf16 terms and bf16 for fp32.
template <typename T> struct weight_frag { using type = frag_f16; };
template <> struct weight_frag<float> { using type = frag_bf16; };
template <typename T> using weight_frag_t = typename weight_frag<T>::type;

// 8 values as the sum of bf16 fragments: three for fp32 (24 bits), one for bf16 queries
// (exact).
template <int N>
__device__ __forceinline__ void split_frag(frag_bf16* f, const float* x) {
    if constexpr (N == 1) {
        pack_frag(f[0], x);
    } else {
        float rest[8];
        frag_bf16 cut;
        pack_frag_hilo(f[0], cut, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] = x[i] - static_cast<float>(f[0].v[i]);
        pack_frag_hilo(f[1], f[2], rest);
    }
}

// 8 probabilities times their powers: three bf16 terms, or fp16, whose rounding (2^-12 of a
// weight at most, against the result's 2^-9) is the one to fewer bits before the result.
template <int N>
__device__ __forceinline__ void split_weights(frag_bf16* f, const float* x) { split_frag<N>(f, x); }
template <int N>
__device__ __forceinline__ void split_weights(frag_f16* f, const float* x) {
    static_assert(N == 1, "one term");
    typedef __attribute__((ext_vector_type(2))) float f32x2_vt;
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2_vt y = {x[2 * i], x[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, f16x2_vt));
    }
    f[0].v = __builtin_bit_cast(f16x8_t, w);
}

// 8 e4m3 codes in fp16 or bf16 (exact).
__device__ __forceinline__ void decode_values(frag_f16& f, uint32_t a, uint32_t b) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;
    u32x4_t w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(a), 1.f, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(a), 1.f, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(b), 1.f, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(b), 1.f, true));
    f.v = __builtin_bit_cast(f16x8_t, w);
}

// 8 e4m3 codes times a power of two, in bf16 (exact).
__device__ __forceinline__ frag_bf16 decode8(uint32_t a, uint32_t b, float power) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;
    u32x4_t w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(a), power, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(a), power, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(b), power, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(b), power, true));
    frag_bf16 f;
    f.v = __builtin_bit_cast(bf16x8_t, w);
    return f;
}

__device__ __forceinline__ void decode_values(frag_bf16& f, uint32_t a, uint32_t b) { f = decode8(a, b, 1.f); }

__device__ __forceinline__ f32x4_t mma16(const frag_bf16& a, const frag_bf16& b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma16(const frag_f16& a, const frag_f16& b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16_t& c, const frag_f16& a, const frag_f16& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.v, b.v, c, 0, 0, 0);
}

__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// 0xff in each byte that is a NaN code (0x7f or 0xff).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
}
constexpr uint32_t ONE_E4M3 = 0x38383838u;     // four codes of 1.0
// NaN for a count above zero, else 0 (by arithmetic: as many masks as there are counts would not
// fit the scalar registers).
__device__ __forceinline__ float nan_if(float count) {
    return count * FLT_MAX * FLT_MAX * 0.f;         // an infinity, or 0, times 0
}
// 0xff in the first n of four bytes.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : (n <= 0 ? 0u : ~0u >> (32 - 8 * n)); }
// Ones for the first a of four tokens and the first b of four more.
__device__ __forceinline__ frag_bf16 shown8(int a, int b) {
    return decode8(first_bytes(a) & ONE_E4M3, first_bytes(b) & ONE_E4M3, 1.f);
}

__device__ __forceinline__ void store4(float* p, const float* x) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store4(bf16_t* p, const float* x) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]));
}

__device__ __forceinline__ int lanes_max(int x) {       // over the 16 rows of a tile
#pragma unroll
    for (int m = 8; m; m >>= 1) x = max(x, __shfl_xor(x, m, 64));
    return x;
}
__device__ __forceinline__ int lanes_min(int x) {
#pragma unroll
    for (int m = 8; m; m >>= 1) x = min(x, __shfl_xor(x, m, 64));
    return x;
}

// What row r of sequence b sees: list positions below this.
__device__ __forceinline__ int row_limit(const attn_args& a, int b, int r) {
    if (r >= a.rows) return 0;
    const int i = r / a.group;
    int cnt = a.n;
    if (a.count) cnt = min(max(a.count[b], 0), a.n);
    if (i >= cnt) return 0;
    const int64_t most = static_cast<int64_t>(a.c.max_pages) * CACHE_TOKENS;
    int64_t len = a.length[b];
    len = len < 0 ? 0 : (len > most ? most : len);
    if (a.causal) len -= cnt - 1 - i;
    return static_cast<int>(len < 0 ? 0 : len);
}

// Both halves' (all four 16-lane groups') maximum of a column.
__device__ __forceinline__ float halves_max(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto y = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float groups_max(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return halves_max(fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
}

// A row's running maximum and sum (base 2).  Weights are 2^(score - m), m = base + lift.
//
// fp16 weights: P = weight times 2^(power - E + 7 + lift).  E is the largest power the wave has
// seen, so that without a lift no P passes 2^15 (weights are at most 2^8).  A row whose weight lies
// on tokens of far smaller powers has P far below: its lift raises those.  `top` is log2 of weight
// times 2^(power - E) at its largest when that was last looked at, or up to 7 less (a look takes the
// powers of a page to be 2^7 below E unless one of them is less), and a lift takes it to 0 from below
// -8.  So the largest P is 2^-1 at least, 2^7 where powers are alike: fp16 keeps 11 bits of every P
// down to 2^-13 (2^-21) of a row's largest, and the error of the others is 2^-24 (2^-32) of that at
// most.
template <bool LIFTED>
struct row_softmax {
    static constexpr float NONE = -FLT_MAX;      // base of a row that has seen nothing
    float base = NONE, l = 0.f, top = 0.f, down = 1.f;     // down: 2^-lift
    __device__ __forceinline__ float lift() const {
        return LIFTED ? static_cast<float>(127 - static_cast<int>(__float_as_uint(down) >> 23)) : 0.f;
    }
    __device__ __forceinline__ float m() const { return base == NONE ? -INFINITY : base + lift(); }
    // The maximum goes to `up`, 2^-E changes by 2^de, some weights times 2^(power - E) are then
    // 2^most: what O is multiplied with.  One factor, since the scales alone may leave fp32.
    __device__ __forceinline__ float move(float up, float de, float most) {
        const float was = lift(), by = base == NONE ? NONE : base + was - up;
        l *= fast_exp2(by);
        if constexpr (!LIFTED) {
            base = up;
            return fast_exp2(by);
        }
        top = fmaxf(top + by + de, most);
        const float now = top < -8.f ? fminf(-floorf(top), 110.f) : 0.f;
        base = up == NONE ? NONE : up - now;
        down = power_of(static_cast<uint32_t>(127 - static_cast<int>(now)));
        return fast_exp2(by + de + (now - was));
    }
};
template <typename T> constexpr bool lifted_of = sizeof(T) == 2;
template <typename T> using row_softmax_t = row_softmax<lifted_of<T>>;

// The exponents (+ 127) of a wave's powers, the same in every lane: the largest so far (E) and what
// it was before the page at hand.  Of the page (or pages) at hand a lane has four bytes, all lanes
// together all of them; `marked` holds the bytes that count, the others 0.
struct powers_seen {
    int most = 0, was = 0;
    // Is one of the marked bytes above E, or more than 2^7 below?
    __device__ __forceinline__ bool news(uint32_t four, uint32_t mask) const {
        return ((four - static_cast<uint32_t>(most - 7) * 0x01010101u) & 0xf8f8f8f8u & mask) != 0;
    }
    // Is one more than 2^by below E?  In any lane.
    __device__ __forceinline__ bool below(uint32_t marked, int by) const {
        bool less = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int byte = static_cast<int>((marked >> (8 * i)) & 0xffu);
            less |= byte != 0 && byte < most - by;
        }
        return __ballot(less) != 0;
    }
    // Brings E up to date; does it change?
    __device__ __forceinline__ bool look(uint32_t marked) {
        const uint32_t ev = max(marked & 0xffu, (marked >> 8) & 0xffu), od = max((marked >> 16) & 0xffu, marked >> 24);
        const int top = static_cast<int>(max(ev, od));
        was = most;
        if (__ballot(top > most) == 0) return false;
        float x = static_cast<float>(top);
        x = fmaxf(x, dpp_f32<0xB1>(x));
        x = fmaxf(x, dpp_f32<0x4E>(x));
        x = fmaxf(x, dpp_f32<0x141>(x));
        x = fmaxf(x, dpp_f32<0x140>(x));
        most = __builtin_amdgcn_readfirstlane(static_cast<int>(groups_max(x)));
        return true;
    }
    // 2^(power - E + 7), of a byte that raised() gave where some are more than 2^134 below
    __device__ __forceinline__ float scaled(uint32_t byte) const {
        return __uint_as_float((byte << 23) + (static_cast<uint32_t>(134 - most) << 23));
    }
    // At least what scaled() gives 0 for.
    __device__ __forceinline__ uint32_t raised(uint32_t byte) const {
        return static_cast<uint32_t>(max(static_cast<int>(byte), most - 134));
    }
    // what takes O back
    __device__ __forceinline__ float back(const row_softmax<true>& w) const {
        return most == 0 ? 0.f : ldexpf(w.down, most - 134);
    }
    __device__ __forceinline__ float back(const row_softmax<false>&) const { return 1.f; }
};

// Valid pages of a list's piece [lo, hi) in order: 64 table entries at a time in
// a register, a bit for each that names a page.
struct page_walk {
    const int32_t* table;
    int at, hi, pages;     // next entries to fetch; pages of the pool
    int ids, base;         // fetched entries (one per lane), their first position
    uint64_t left;         // of those, still to visit

    __device__ __forceinline__ page_walk(const int32_t* t, int lo, int hi_, int n)
        : table(t), at(lo), hi(hi_), pages(n), ids(-1), base(lo), left(0) {}
    // `mine`: which of 64 entries in a row the caller visits
    __device__ __forceinline__ void fetch(uint64_t mine) {
        const int x = at + lane_id();
        start(x < hi ? table[x] : -1, mine);
    }
    // the same with the entries at hand (lane i: entry at + i, whatever it is past hi)
    __device__ __forceinline__ void start(int entry, uint64_t mine) {
        ids = at + lane_id() < hi ? entry : -1;
        left = __ballot(ids >= 0 && ids < pages) & mine;
        base = at;
        at += 64;
    }
    // position and page of the next one; false at the end
    __device__ __forceinline__ bool next(int& pos, int& id, uint64_t mine = ~0ull) {
        while (left == 0) {
            if (at >= hi) return false;
            fetch(mine);
        }
        const int bit = __builtin_ctzll(left);
        left &= left - 1;
        pos = base + bit;
        id = __builtin_amdgcn_readlane(ids, bit);
        return true;
    }
};

// The piece of a list, and its row tile, that a workgroup takes.  The tiles of a
// piece run on one XCD, whose L2 then holds the piece's pages.  Spread: next pieces
// on next XCDs, so that the long and the short sequences of a batch load all of
// them alike (16 sequences of 20,000 to 76,800 tokens: 287 us against 332 with
// neighbouring lists on one XCD, 16 x 8 lists of 200 rows 275 against 327); else a
// run of pieces for every XCD, which keeps a few pieces of many tiles even (12 lists
// of 1,792 rows: 434 us against 590 spread).
__device__ __forceinline__ uint32_t piece_of(const attn_args& a, int& tile) {
    if (!a.spread) {
        const uint32_t item = static_cast<uint32_t>(xcd_item(blockIdx.x, gridDim.x));
        tile = static_cast<int>(item % a.tiles);
        return item / a.tiles;
    }
    const uint32_t turn = blockIdx.x >> 3, t = turn / a.tiles;
    tile = static_cast<int>(turn - t * a.tiles);
    return t * 8 + (blockIdx.x & 7);
}

__device__ __forceinline__ const int32_t* list_of(const attn_args& a, int b, int h) {
    return a.c.table + (static_cast<int64_t>(b) * a.c.table_heads + (a.c.table_heads > 1 ? h : 0)) * a.c.max_pages;
}

// One row tile's state in one wave: its running maximum and sum (base 2) and
// O^T, rows d = 16 c + 4 g + i, column lane % 16.
template <typename T, int D>
struct tile_state {
    row_softmax_t<T> w;
    f32x4_t o[D / 16];
};

// A lane's share of a page: K's codes of 16 t + lane % 16 and V's, and their powers.
template <int D>
struct page_data {
    uint4 k[4 * (D / 64)], v[D / 16], ve;
    uint32_t ke;
};
template <int D>
__device__ __forceinline__ void load_page(page_data<D>& pd, const char* page) {
    const int lane = lane_id();
    const uint4* kp = reinterpret_cast<const uint4*>(page) + lane;
    const uint4* vp = reinterpret_cast<const uint4*>(page + 64 * D) + lane;
#pragma unroll
    for (int i = 0; i < 4 * (D / 64); ++i) pd.k[i] = kp[i * 64];
    pd.ke = *reinterpret_cast<const uint32_t*>(page + 128 * D + (lane & 15) * 4);
    pd.ve = *reinterpret_cast<const uint4*>(page + 128 * D + 64 + (lane >> 4) * 16);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) pd.v[i] = vp[i * 64];
    // all of them requested before the first is waited for
    __builtin_amdgcn_sched_barrier(0);
}

// One page for XT tiles, decoded once for all of them.  MASKED: some row's limit,
// or the list's end, may lie inside it.
template <typename T, int D, int XT, bool MASKED>
__device__ __forceinline__ void page_step(const page_data<D>& pd, const char* page, int pos, const int (&limit)[XT], int lim_max,
                                          const frag_bf16 (&qf)[XT][D / 32][terms_of<T>], float scale,
                                          tile_state<T, D> (&st)[XT], powers_seen& seen) {
    constexpr int NT = terms_of<T>;
    const int g = lane_id() >> 4;
    f32x4_t s[XT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const float power = power_of((pd.ke >> (8 * t)) & 0xffu);
#pragma unroll
        for (int x = 0; x < XT; ++x) s[x][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
            const uint4 w = pd.k[t * (D / 64) + u];
            const frag_bf16 k0 = decode8(w.x, w.y, power), k1 = decode8(w.z, w.w, power);
#pragma unroll
            for (int y = NT - 1; y >= 0; --y)
#pragma unroll
                for (int x = 0; x < XT; ++x) {
                    s[x][t] = mma16(k0, qf[x][2 * u][y], s[x][t]);
                    s[x][t] = mma16(k1, qf[x][2 * u + 1][y], s[x][t]);
                }
        }
    }
    uint32_t vw[4] = {pd.ve.x, pd.ve.y, pd.ve.z, pd.ve.w};
    uint4 vr[D / 16];
#pragma unroll
    for (int c = 0; c < D / 16; ++c) vr[c] = pd.v[c];
    weight_frag_t<T> pf[XT][2][NT];
    // a quarter of the lane's tokens' powers, of those below lim_max
    const int at = lane_id() & 3;
    const uint32_t four = at & 2 ? (at & 1 ? vw[3] : vw[2]) : (at & 1 ? vw[1] : vw[0]);
    uint32_t marked = ~0u;
    if constexpr (MASKED) marked = first_bytes(lim_max - (pos + 16 * at + 4 * g));
    float mx[XT];
    const bool news = NT == 1 && seen.news(four, marked);
    bool far = false;
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        if constexpr (MASKED) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (pos + 16 * t + 4 * g + i >= limit[x]) s[x][t][i] = -INFINITY;
        }
        mx[x] = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; i += 2) mx[x] = fmaxf(fmaxf(mx[x], s[x][t][i]), s[x][t][i + 1]);
        mx[x] = groups_max(mx[x]);
        far |= fmaf(mx[x], scale, -st[x].w.base) > 8.f;
    }
    // the running maxima move only when one would grow by more than 8 (weights
    // up to 2^8 of the first), less with a lift: most pages leave O alone
    if (__ballot(far || news) != 0) {
        bool moves = __ballot(far) != 0;
        if constexpr (NT == 1) {
            moves |= seen.look(four & marked);
            if (seen.below(four & marked, 134)) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    uint32_t w = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w |= seen.raised((vw[t] >> (8 * i)) & 0xffu) << (8 * i);
                    vw[t] = w;
                }
            }
        }
        const bool wide = NT == 1 && moves && seen.below(four & marked, 7);
#pragma unroll
        for (int x = 0; x < XT; ++x) {
            if (!moves) continue;
            row_softmax_t<T>& w = st[x].w;
            const float up = fmaxf(w.base + w.lift(), mx[x] * scale);
            float most = fmaf(mx[x], scale, -up) - 7.f;
            if (wide) {
                most = -INFINITY;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        most = fmaxf(most, fmaf(s[x][t][i], scale, -up) +
                                               static_cast<float>(static_cast<int>((vw[t] >> (8 * i)) & 0xffu) - seen.most));
                most = groups_max(most);
            }
            const float f = w.move(up, static_cast<float>(seen.was - seen.most), most);
#pragma unroll
            for (int c = 0; c < D / 16; ++c) st[x].o[c] *= f;
        }
    }
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        row_softmax_t<T>& w = st[x].w;
        float p[4][4], sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = fast_exp2(fmaf(s[x][t][i], scale, -w.base));
                sum += e;
                // a masked place's power may be anything
                const uint32_t byte = (vw[t] >> (8 * i)) & 0xffu;
                p[t][i] = MASKED && e == 0.f ? 0.f : e * (NT == 1 ? seen.scaled(byte) : power_of(byte));
            }
        w.l = fmaf(sum, w.down, w.l);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const float z[8] = {p[2 * y][0], p[2 * y][1], p[2 * y][2], p[2 * y][3],
                                p[2 * y + 1][0], p[2 * y + 1][1], p[2 * y + 1][2], p[2 * y + 1][3]};
            split_weights<NT>(pf[x][y], z);
        }
    }
    uint32_t keep[4], any = 0;
    if constexpr (MASKED) {
        // Codes past every row's limit are whatever the page held: taken as
        // zeros.  A NaN below it, which some rows see and others do not, is
        // taken out of the product, too.
#pragma unroll
        for (int t = 0; t < 4; ++t) keep[t] = first_bytes(lim_max - (pos + 16 * t + 4 * g));
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            uint32_t w[4] = {vr[c].x & keep[0], vr[c].y & keep[1], vr[c].z & keep[2], vr[c].w & keep[3]};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t nan = nan_bytes(w[t]);
                w[t] &= ~nan;
                any |= nan;
            }
            vr[c] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        weight_frag_t<T> v0, v1;
        decode_values(v0, vr[c].x, vr[c].y);
        decode_values(v1, vr[c].z, vr[c].w);
#pragma unroll
        for (int y = NT - 1; y >= 0; --y)
#pragma unroll
            for (int x = 0; x < XT; ++x) {
                st[x].o[c] = mma16(v0, pf[x][0][y], st[x].o[c]);
                st[x].o[c] = mma16(v1, pf[x][1][y], st[x].o[c]);
            }
    }
    if constexpr (MASKED) {
        // A NaN goes to the rows that see it, whatever their weight on it: a second product,
        // from the page's codes once more, counts it where a row's limit lies past it.
        if (__ballot(any != 0) == 0) return;
        const uint4* vp = reinterpret_cast<const uint4*>(page + 64 * D) + lane_id();
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            const uint4 v = vp[c * 64];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t nan[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) nan[t] = nan_bytes(w[t] & keep[t]) & ONE_E4M3;
#pragma unroll
            for (int x = 0; x < XT; ++x) {
                const int here = limit[x] - (pos + 4 * g);
                f32x4_t hit = f32x4_t{0.f, 0.f, 0.f, 0.f};
                hit = mma16(decode8(nan[0], nan[1], 1.f), shown8(here, here - 16), hit);
                hit = mma16(decode8(nan[2], nan[3], 1.f), shown8(here - 32, here - 48), hit);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    st[x].o[c][i] += nan_if(hit[i]);
            }
        }
    }
}

// Element offset of row r (query head and token of KV head h) in q or o.
__device__ __forceinline__ int64_t row_offset(const row_view& v, const attn_args& a, int b, int h, int r) {
    const int i = r / a.group, hg = r - i * a.group;
    return b * v.batch + static_cast<int64_t>(h * a.group + hg) * v.head + static_cast<int64_t>(i) * v.token;
}
__device__ __forceinline__ void store_lse(const attn_args& a, int b, int h, int r, float base, float l) {
    const int i = r / a.group, hg = r - i * a.group;
    a.lse[(static_cast<int64_t>(b) * a.c.heads * a.group + h * a.group + hg) * a.n + i] = (base + log2f(l)) * LN2;
}

// Few rows: WAVES waves take turns at the list's pages, each for all the rows
// (XT tiles of 16).  Two waves a SIMD at D = 128, also where the registers would hold
// three: plan_attn cuts lists for that (16 x 8 lists of 20,000 to 76,800 tokens: 280 us
// against 290).
template <typename T, int D, int WAVES, int XT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, D == 128 ? 2 : 4))) void attn_cache_kernel(
    attn_args a) {
    constexpr int NT = terms_of<T>, TR = XT * TILE;
    __shared__ float so[WAVES][TR][D + 4];
    __shared__ float sml[WAVES][TR][2];
    const int lane = lane_id(), wave = wave_id(), g = lane >> 4, col = lane & 15;
    int tile;
    const uint32_t item = piece_of(a, tile);
    if (item >= a.pieces) return;
    const int split = static_cast<int>(item % a.splits);
    const uint32_t bh = item / a.splits;
    const int b = static_cast<int>(bh / a.c.heads), h = static_cast<int>(bh % a.c.heads);
    // a list in one piece starts at its first entry: fetched beside the lengths
    uint64_t mine = 0;
#pragma unroll
    for (int i = 0; i < 64; i += WAVES) mine |= 1ull << i;
    mine <<= wave;
    const int32_t* list = list_of(a, b, h);
    const int early = a.splits == 1 && lane < a.c.max_pages ? list[lane] : -1;
    // rows that see nothing take what the others compute and drop it at the end
    int limit[XT], most = 0, least = INT32_MAX;
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        limit[x] = row_limit(a, b, tile * TR + x * TILE + col);
        most = max(most, limit[x]);
        least = limit[x] > 0 ? min(least, limit[x]) : least;
    }
    const int lim_max = __builtin_amdgcn_readfirstlane(lanes_max(most));
    const int lim_min = __builtin_amdgcn_readfirstlane(lanes_min(least));
    const int pages = (lim_max + CACHE_TOKENS - 1) / CACHE_TOKENS;
    const int lo = static_cast<int>(static_cast<int64_t>(pages) * split / a.splits);
    const int hi = static_cast<int>(static_cast<int64_t>(pages) * (split + 1) / a.splits);
    page_walk walk(list, lo, hi, a.c.pages);
    if (a.splits == 1) walk.start(early, mine);
    else if (lo < hi) walk.fetch(mine);

    frag_bf16 qf[XT][D / 32][NT];
    tile_state<T, D> st[XT];
    powers_seen seen;
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        const int r = tile * TR + x * TILE + col;
        const T* q = static_cast<const T*>(a.q.ptr) + (r < a.rows ? row_offset(a.q, a, b, h, r) : 0);
#pragma unroll
        for (int u = 0; u < D / 32; ++u) {
            float y[8] = {};
            if (r < a.rows) {
                const T* e = q + (u / 2) * 64 + g * 16 + (u & 1) * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = to_f32(e[i]);
            }
            split_frag<NT>(qf[x][u], y);
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) st[x].o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float scale = LOG2E / sqrtf(static_cast<float>(D));
    int pg, id;
    bool more = walk.next(pg, id, mine);
    const auto page = [&]() { return a.c.pool + (static_cast<int64_t>(id) * a.c.heads + h) * cache_page_bytes(D); };
    const auto whole = [&]() { return more && (pg + 1) * CACHE_TOKENS <= lim_min; };
    for (; whole(); more = walk.next(pg, id, mine)) {
        page_data<D> x;
        load_page<D>(x, page());
        page_step<T, D, XT, false>(x, nullptr, 0, limit, lim_max, qf, scale, st, seen);
    }
    for (; more; more = walk.next(pg, id, mine)) {
        page_data<D> x;
        load_page<D>(x, page());
        page_step<T, D, XT, true>(x, page(), pg * CACHE_TOKENS, limit, lim_max, qf, scale, st, seen);
    }
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        float l = st[x].w.l;
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        const bool dead = limit[x] == 0;
        const int row = x * TILE + col;
        const float back = seen.back(st[x].w);
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            *reinterpret_cast<f32x4_t*>(&so[wave][row][16 * c + 4 * g]) =
                dead ? f32x4_t{0.f, 0.f, 0.f, 0.f} : st[x].o[c] * back;
        if (g == 0) {
            sml[wave][row][0] = dead ? -INFINITY : st[x].w.m();
            sml[wave][row][1] = dead ? 0.f : l;
        }
    }
    __syncthreads();
    // join the waves: a thread takes 4 elements of a row
    for (int at = threadIdx.x; at < TR * (D / 4); at += 64 * WAVES) {
        const int row = at / (D / 4), d0 = at % (D / 4) * 4, rr = tile * TR + row;
        if (rr >= a.rows) continue;
        float m = sml[0][row][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sml[w][row][0]);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f, o[4] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = fast_exp2(sml[w][row][0] - base);
            const float4 y = *reinterpret_cast<const float4*>(&so[w][row][d0]);
            l += f * sml[w][row][1];
            o[0] += f * y.x;
            o[1] += f * y.y;
            o[2] += f * y.z;
            o[3] += f * y.w;
        }
        if (a.splits > 1) {
            float* part = a.part + ((static_cast<int64_t>(bh) * a.tiles + tile) * a.splits + split) * (TR * (D + 2));
            store4(part + row * D + d0, o);
            if (d0 == 0) {
                part[TR * D + 2 * row] = m;
                part[TR * D + 2 * row + 1] = l;
            }
            continue;
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = l == 0.f ? 0.f : o[i] * inv;
        store4(static_cast<T*>(a.o.ptr) + row_offset(a.o, a, b, h, rr) + d0, o);
        if (d0 == 0) store_lse(a, b, h, rr, base, l);
    }
}

// ---------------------------------------------------------------------------
// Many rows: a wave takes 32 of them on 32x32x16 MFMAs, a workgroup's four waves
// walk the same pages, copied into LDS asynchronously one page ahead.
//
// The page's order fits these fragments too: lane (half h, r = lane % 32) takes
// K's 16-byte piece 2 w + h of token 32 T + r for two k-steps, and V's pieces
// g = h and h + 2 of element 32 c + r, whose dwords t are the two runs of four
// tokens that the accumulators of S^T hold for k-step t.  Reads are runs of
// 256 bytes per 16 lanes: no bank conflicts, no padding, one address per lane.
// ---------------------------------------------------------------------------
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;

template <int D>
__device__ __forceinline__ void copy_page(char* lds, const char* page, int wave, int lane) {
    // 128 D bytes of codes: each wave 32 D of them in whole 1 KB copies
    constexpr int NR = D / 32;
    const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void_t*)lds)) + wave * 32 * D;
    const int from = wave * 32 * D + lane * 16 + DMA_BIAS;
    const int off[4] = {from, from, from, from};      // the copies' own offsets step both sides
    dma16_run<NR>(to, reinterpret_cast<uint64_t>(page) - DMA_BIAS, off);
}

// A wave's 32 rows: running maximum and sum (base 2), O^T of column lane % 32,
// elements 32 c + 8 (i / 4) + 4 (lane / 32) + i % 4.
template <typename T, int D>
struct rows_state {
    row_softmax_t<T> w;
    f32x16_t o[D / 32];
};

// Moves the running maximum, and the scale of P, for the scores s of N / 2 pages, whose powers
// are power[page][1]; `mx` is their largest.  Most pages leave O alone: see page_step.
template <typename T, int D, int N>
__device__ __forceinline__ void rows_move(const f32x16_t (&s)[N], const float (*power)[2][64], float mx, float scale,
                                          powers_seen& seen, rows_state<T, D>& st) {
    constexpr bool LIFTED = lifted_of<T>;
    bool far = fmaf(mx, scale, -st.w.base) > 8.f;
    if constexpr (LIFTED) far |= seen.was != seen.most;
    if (__ballot(far) == 0) return;
    const float up = fmaxf(st.w.base + st.w.lift(), mx * scale);
    float most = fmaf(mx, scale, -up) - 7.f;
    bool wide = false;          // a lane's token of each page more than 2^7 below E (past a limit: whatever)
    if constexpr (LIFTED) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) wide |= power[i][1][lane_id()] < 1.f;
        wide = __ballot(wide) != 0;
    }
    if (wide) {
        const int h2 = lane_id() >> 5;
        most = -INFINITY;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float pw = power[t / 2][1][(t % 2) * 32 + 8 * (i / 4) + 4 * h2 + i % 4];
                most = fmaxf(most, fmaf(s[t][i], scale, -up) + static_cast<float>(static_cast<int>(__float_as_uint(pw) >> 23) - 134));
            }
        most = halves_max(most);
    }
    const float f = st.w.move(up, static_cast<float>(seen.was - seen.most), most);
    seen.was = seen.most;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[c][i] *= f;
}

// One page in LDS for a wave's rows, where some row's limit, or the list's end,
// may lie inside it.
template <typename T, int D>
__device__ __forceinline__ void rows_step(const char* kp, const char* vp, const float (*page_power)[2][64], int first,
                                          int limit, int wmax, const frag_bf16 (&qf)[D / 32][2][terms_of<T>],
                                          float scale, powers_seen& seen, rows_state<T, D>& st) {
    const float (*power)[64] = *page_power;
    constexpr int NT = terms_of<T>, KC = D / 32, VC = D / 32;
    const int lane = lane_id(), h2 = lane >> 5, col = lane & 31;
    f32x16_t s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
        const float pw = power[0][t * 32 + col];
#pragma unroll
        for (int w = 0; w < KC; ++w) {
            const uint4 x = *reinterpret_cast<const uint4*>(kp + t * 2 * (D / 64) * 1024 + (w / 2) * 1024 + (w % 2) * 512);
            const frag_bf16 k0 = decode8(x.x, x.y, pw), k1 = decode8(x.z, x.w, pw);
#pragma unroll
            for (int y = NT - 1; y >= 0; --y) {
                mma(s[t], k0, qf[w][0][y]);
                mma(s[t], k1, qf[w][1][y]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (first + t * 32 + 8 * (i / 4) + 4 * h2 + i % 4 >= limit) s[t][i] = -INFINITY;
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[t][i]), s[t][i + 1]);
    mx = halves_max(mx);
    rows_move<T, D>(s, page_power, mx, scale, seen, st);
    float sum = 0.f;
    weight_frag_t<T> pf[4][NT];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = fast_exp2(fmaf(s[t / 2][(t % 2) * 8 + i], scale, -st.w.base));
            sum += y[i];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const float4 pw = *reinterpret_cast<const float4*>(&power[1][t * 16 + x * 8 + 4 * h2]);
            const float pv[4] = {pw.x, pw.y, pw.z, pw.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // a masked place's power may be anything
                y[4 * x + i] = y[4 * x + i] == 0.f ? 0.f : y[4 * x + i] * pv[i];
            }
        }
        split_weights<NT>(pf[t], y);
    }
    st.w.l = fmaf(sum, st.w.down, st.w.l);
    uint32_t keep[4][2], any = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x) keep[t][x] = first_bytes(wmax - (first + 16 * t + 8 * x + 4 * h2));
    // as in page_step: stale codes are zeros, a NaN goes to the rows that see it
#pragma unroll
    for (int c = 0; c < VC; ++c) {
        const uint4 va = *reinterpret_cast<const uint4*>(vp + c * 2048);
        const uint4 vb = *reinterpret_cast<const uint4*>(vp + c * 2048 + 512);
        uint32_t w[4][2] = {{va.x, vb.x}, {va.y, vb.y}, {va.z, vb.z}, {va.w, vb.w}};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                w[t][x] &= keep[t][x];
                const uint32_t nan = nan_bytes(w[t][x]);
                w[t][x] &= ~nan;
                any |= nan;
            }
            weight_frag_t<T> vf;
            decode_values(vf, w[t][0], w[t][1]);
#pragma unroll
            for (int z = NT - 1; z >= 0; --z) mma(st.o[c], vf, pf[t][z]);
        }
    }
    if (__ballot(any != 0) == 0) return;
#pragma unroll
    for (int c = 0; c < VC; ++c) {
        const uint4 va = *reinterpret_cast<const uint4*>(vp + c * 2048);
        const uint4 vb = *reinterpret_cast<const uint4*>(vp + c * 2048 + 512);
        const uint32_t w[4][2] = {{va.x, vb.x}, {va.y, vb.y}, {va.z, vb.z}, {va.w, vb.w}};
        f32x16_t hit;
#pragma unroll
        for (int i = 0; i < 16; ++i) hit[i] = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int here = limit - (first + 16 * t + 4 * h2);
            mma(hit, decode8(nan_bytes(w[t][0] & keep[t][0]) & ONE_E4M3, nan_bytes(w[t][1] & keep[t][1]) & ONE_E4M3, 1.f),
                shown8(here, here - 8));
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            st.o[c][i] += nan_if(hit[i]);
    }
}

// The two pages of a stage together, no limit inside either.
template <typename T, int D>
__device__ __forceinline__ void rows_pair(const char* lds, int kbase, int vbase, const float (*power)[2][64],
                                          const frag_bf16 (&qf)[D / 32][2][terms_of<T>], float scale, powers_seen& seen,
                                          rows_state<T, D>& st) {
    constexpr int NT = terms_of<T>, KC = D / 32, VC = D / 32;
    const int lane = lane_id(), h2 = lane >> 5, col = lane & 31;
    f32x16_t s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const char* kp = lds + (t / 2) * 128 * D + kbase;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
        const float pw = power[t / 2][0][(t % 2) * 32 + col];
#pragma unroll
        for (int w = 0; w < KC; ++w) {
            const uint4 x = *reinterpret_cast<const uint4*>(kp + (t % 2) * 2 * (D / 64) * 1024 + (w / 2) * 1024 + (w % 2) * 512);
            const frag_bf16 k0 = decode8(x.x, x.y, pw), k1 = decode8(x.z, x.w, pw);
#pragma unroll
            for (int y = NT - 1; y >= 0; --y) {
                mma(s[t], k0, qf[w][0][y]);
                mma(s[t], k1, qf[w][1][y]);
            }
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[t][i]), s[t][i + 1]);
    mx = halves_max(mx);
    rows_move<T, D>(s, power, mx, scale, seen, st);
    float l2[2] = {0.f, 0.f};
#pragma unroll
    for (int pg = 0; pg < 2; ++pg) {
        const char* vp = lds + pg * 128 * D + vbase;
        weight_frag_t<T> pf[4][NT];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = fast_exp2(fmaf(s[2 * pg + t / 2][(t % 2) * 8 + i], scale, -st.w.base));
                l2[i & 1] += y[i];
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float4 pw = *reinterpret_cast<const float4*>(&power[pg][1][t * 16 + x * 8 + 4 * h2]);
                const float pv[4] = {pw.x, pw.y, pw.z, pw.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) y[4 * x + i] *= pv[i];
            }
            split_weights<NT>(pf[t], y);
        }
#pragma unroll
        for (int c = 0; c < VC; ++c) {
            const uint4 va = *reinterpret_cast<const uint4*>(vp + c * 2048);
            const uint4 vb = *reinterpret_cast<const uint4*>(vp + c * 2048 + 512);
            const uint32_t w[4][2] = {{va.x, vb.x}, {va.y, vb.y}, {va.z, vb.z}, {va.w, vb.w}};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                weight_frag_t<T> vf;
            decode_values(vf, w[t][0], w[t][1]);
#pragma unroll
                for (int z = NT - 1; z >= 0; --z) mma(st.o[c], vf, pf[t][z]);
            }
        }
    }
    st.w.l = fmaf(l2[0] + l2[1], st.w.down, st.w.l);
}

template <typename T, int D>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 4 ? 1 : 2) void attn_cache_rows_kernel(attn_args a) {
    constexpr int NT = terms_of<T>, KC = D / 32, VC = D / 32;
    __shared__ __attribute__((aligned(1024))) char codes[2][STAGE][128 * D];
    __shared__ __attribute__((aligned(16))) float power[NW][STAGE][2][64];
    const int lane = lane_id(), wave = wave_id(), h2 = lane >> 5, col = lane & 31;
    int tile;
    const uint32_t item = piece_of(a, tile);
    if (item >= a.pieces) return;
    const int split = static_cast<int>(item % a.splits);
    const uint32_t bh = item / a.splits;
    const int b = static_cast<int>(bh / a.c.heads), h = static_cast<int>(bh % a.c.heads);
    const int r = tile * ROWS + wave * 32 + col;
    const int limit = row_limit(a, b, r);
    // the rows' limits: the wave's largest, the workgroup's largest and (of rows that see something,
    // the others drop what they compute at the end) smallest
    int wmax = limit, wmin = limit > 0 ? limit : INT32_MAX;
#pragma unroll
    for (int m = 16; m; m >>= 1) {
        wmin = min(wmin, __shfl_xor(wmin, m, 64));
        wmax = max(wmax, __shfl_xor(wmax, m, 64));
    }
    wmax = __builtin_amdgcn_readfirstlane(wmax);
    __shared__ int ends[NW][2];
    if (lane == 0) {
        ends[wave][0] = wmin;
        ends[wave][1] = wmax;
    }
    __syncthreads();
    int all = 0, full = INT32_MAX;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        full = min(full, ends[w][0]);
        all = max(all, ends[w][1]);
    }
    all = __builtin_amdgcn_readfirstlane(all);
    full = __builtin_amdgcn_readfirstlane(full) / CACHE_TOKENS;     // pages before this one need no mask
    const int pages = (all + CACHE_TOKENS - 1) / CACHE_TOKENS;
    const int lo = static_cast<int>(static_cast<int64_t>(pages) * split / a.splits);
    const int hi = static_cast<int>(static_cast<int64_t>(pages) * (split + 1) / a.splits);

    frag_bf16 qf[KC][2][NT];
    const T* q = static_cast<const T*>(a.q.ptr) + (r < a.rows ? row_offset(a.q, a, b, h, r) : 0);
#pragma unroll
    for (int w = 0; w < KC; ++w)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            float y[8] = {};
            if (r < a.rows) {
                const T* e = q + (2 * w + h2) * 16 + z * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = to_f32(e[i]);
            }
            split_frag<NT>(qf[w][z], y);
        }
    rows_state<T, D> st;
    powers_seen seen;
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[c][i] = 0.f;
    const float scale = LOG2E / sqrtf(static_cast<float>(D));
    const int kbase = (col >> 4) * (D / 64) * 1024 + h2 * 256 + (col & 15) * 16;
    const int vbase = 64 * D + (col >> 4) * 1024 + h2 * 256 + (col & 15) * 16;
    // in-page places of this lane's token's two powers
    const int ke_at = 128 * D + (lane & 15) * 4 + (lane >> 4);
    const int ve_at = 128 * D + 64 + ((lane >> 2) & 3) * 16 + (lane >> 4) * 4 + (lane & 3);

    page_walk walk(list_of(a, b, h), lo, hi, a.c.pages);
    int pos[STAGE], buf = 0, have = 0;
    uint8_t ke[STAGE] = {}, ve[STAGE] = {};
    auto request = [&](int to) {
        have = 0;
#pragma unroll
        for (int x = 0; x < STAGE; ++x) {
            int id;
            pos[x] = 0;
            if (have < x || !walk.next(pos[x], id)) continue;
            const char* page = a.c.pool + (static_cast<int64_t>(id) * a.c.heads + h) * cache_page_bytes(D);
            ke[x] = static_cast<uint8_t>(page[ke_at]);
            ve[x] = static_cast<uint8_t>(page[ve_at]);
            copy_page<D>(codes[to][x], page, wave, lane);
            have = x + 1;
        }
    };
    request(0);
    // Waits for the pages at hand, requests the next ones and says which were at
    // hand.  Past the barrier every wave is done with the other buffer.
    int at[STAGE];
    auto turn = [&]() {
        if constexpr (NT == 1) {
            uint32_t marked = 0;
#pragma unroll
            for (int x = 0; x < STAGE; ++x)
                if (x < have && pos[x] * CACHE_TOKENS + lane < wmax) marked |= static_cast<uint32_t>(ve[x]) << (8 * x);
            seen.look(marked);
        }
#pragma unroll
        for (int x = 0; x < STAGE; ++x) {
            power[wave][x][0][lane] = power_of(ke[x]);
            power[wave][x][1][lane] = NT == 1 ? seen.scaled(seen.raised(ve[x])) : power_of(ve[x]);
            at[x] = pos[x];
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        wg_barrier();
        const int n = have;
        request(buf ^ 1);
        return n;
    };
    while (have == STAGE && pos[STAGE - 1] < full) {
        turn();
        rows_pair<T, D>(codes[buf][0], kbase, vbase, power[wave], qf, scale, seen, st);
        buf ^= 1;
    }
    while (have > 0) {
        const int n = turn();
#pragma unroll 1
        for (int x = 0; x < n; ++x) {
            const int first = (x ? at[STAGE - 1] : at[0]) * CACHE_TOKENS;
            if (first < wmax)
                rows_step<T, D>(codes[buf][x] + kbase, codes[buf][x] + vbase, &power[wave][x], first, limit, wmax, qf,
                                      scale, seen, st);
        }
        buf ^= 1;
    }
    f32x16_t(&o)[VC] = st.o;
    float m = st.w.m(), l = st.w.l;
    const float back = seen.back(st.w);
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= back;
    l += swap_half(l);
    if (limit == 0) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    }
    const float base = m == -INFINITY ? 0.f : m;
    if (r >= a.rows) return;
    if (a.splits > 1) {
        float* part = a.part + ((static_cast<int64_t>(bh) * a.tiles + tile) * a.splits + split) * (ROWS * (D + 2));
        const int row = wave * 32 + col;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float x[4] = {o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]};
                store4(part + row * D + c * 32 + 2 * i + 4 * h2, x);
            }
        if (h2 == 0) {
            part[ROWS * D + 2 * row] = m;
            part[ROWS * D + 2 * row + 1] = l;
        }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = static_cast<T*>(a.o.ptr) + row_offset(a.o, a, b, h, r);
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float x[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) x[y] = l == 0.f ? 0.f : o[c][i + y] * inv;
            store4(out + c * 32 + 2 * i + 4 * h2, x);
        }
    if (h2 == 0) store_lse(a, b, h, r, base, l);
}

// Joins the pieces of a row tile.  A row is joined by SLICES groups of 32 lanes,
// each taking every SLICES-th piece, whose sums are added in order: one group
// (8 rows a workgroup) for up to 8 pieces, eight groups for up to 32, 32 for more,
// where a group's loads one after the other took longer than the pieces themselves
// (512 pieces of one row: the whole call 41.4 us with eight groups, 29.1 with 32).
template <typename T, int D, int SLICES>
__global__ __launch_bounds__(SLICES > 8 ? 32 * SLICES : 256) void attn_cache_join_kernel(attn_args a, int tile_rows) {
    constexpr int RPW = SLICES > 8 ? 1 : 8 / SLICES;       // rows of a workgroup
    __shared__ float so[SLICES > 1 ? SLICES : 1][D], sl[SLICES];
    const int64_t stride = static_cast<int64_t>(tile_rows) * (D + 2);
    const int subs = tile_rows / RPW;
    const uint32_t item = blockIdx.x / subs, bh = item / a.tiles;
    const int tile = static_cast<int>(item % a.tiles), sub = static_cast<int>(blockIdx.x % subs);
    const int b = static_cast<int>(bh / a.c.heads), h = static_cast<int>(bh % a.c.heads);
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, slice = group % SLICES;
    const int row = sub * RPW + group / SLICES, rr = tile * tile_rows + row;
    if (rr >= a.rows) return;             // all lanes of a row together (SLICES > 1: the workgroup)
    const float* part = a.part + static_cast<int64_t>(item) * a.splits * stride;
    const float* ml = part + static_cast<int64_t>(tile_rows) * D + 2 * row;
    float m = -INFINITY;
    for (int x = lane; x < a.splits; x += 32) m = fmaxf(m, ml[x * stride]);
#pragma unroll
    for (int k = 16; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k, 64));
    const float base = m == -INFINITY ? 0.f : m;
    float l = 0.f, o[D / 32] = {};
    // 32 of this slice's pieces at a time: their weights one a lane, then their sums
    for (int x0 = slice; x0 < a.splits; x0 += 32 * SLICES) {
        float f = 0.f;
        if (x0 + lane * SLICES < a.splits) {
            const float2 y = *reinterpret_cast<const float2*>(ml + (x0 + lane * SLICES) * stride);
            f = fast_exp2(y.x - base);
            l += f * y.y;
        }
        const int n = min(32, (a.splits - x0 + SLICES - 1) / SLICES);
        const float* px = part + x0 * stride + row * D + lane * (D / 32);
#pragma unroll 4
        for (int x = 0; x < n; ++x) {
            const float w = __shfl(f, (threadIdx.x & 32) + x, 64);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) o[i] += w * px[x * SLICES * stride + i];
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
    T* out = static_cast<T*>(a.o.ptr) + row_offset(a.o, a, b, h, rr) + lane * (D / 32);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) from_f32(out[i], l == 0.f ? 0.f : o[i] * inv);
    if (lane == 0) store_lse(a, b, h, rr, base, l);
}

// How a call is cut: rows per workgroup and its waves, row tiles of a KV head,
// pieces of a list.
struct attn_plan {
    int tile_rows, waves;
    int64_t tiles;
    int splits;
};

// fp32 rows of D = 128 take three times the registers: a pair of tiles would not fit.
template <typename T, int D> constexpr bool two_tiles = !(sizeof(T) == 4 && D == 128);

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

}  // namespace

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

namespace {

template <typename T, int D>
void launch_attn(const attn_args& a, const attn_plan& p, hipStream_t s) {
    const int64_t items = static_cast<int64_t>(a.c.batch) * a.c.heads * p.tiles;
    const int64_t pieces = a.spread ? (static_cast<int64_t>(a.pieces) + 7) / 8 * 8 : a.pieces;
    const dim3 grid(static_cast<unsigned>(pieces * p.tiles)), block(64 * p.waves);
    if (p.tile_rows == ROWS) hipLaunchKernelGGL((attn_cache_rows_kernel<T, D>), grid, block, 0, s, a);
    else if (p.tile_rows == TILE) {
        if (p.waves == 8) hipLaunchKernelGGL((attn_cache_kernel<T, D, 8, 1>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((attn_cache_kernel<T, D, 4, 1>), grid, block, 0, s, a);
    } else if constexpr (two_tiles<T, D>) {
        if (p.waves == 8) hipLaunchKernelGGL((attn_cache_kernel<T, D, 8, 2>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((attn_cache_kernel<T, D, 4, 2>), grid, block, 0, s, a);
    }
    const auto rows_of = [&](int per_wg) { return dim3(static_cast<unsigned>(items * (p.tile_rows / per_wg))); };
    if (p.splits > 32)
        hipLaunchKernelGGL((attn_cache_join_kernel<T, D, 32>), rows_of(1), dim3(1024), 0, s, a, p.tile_rows);
    else if (p.splits > 8)
        hipLaunchKernelGGL((attn_cache_join_kernel<T, D, 8>), rows_of(1), dim3(256), 0, s, a, p.tile_rows);
    else if (p.splits > 1)
        hipLaunchKernelGGL((attn_cache_join_kernel<T, D, 1>), rows_of(8), dim3(256), 0, s, a, p.tile_rows);
}

}  // namespace

hipError_t launch_attn_cache(int dtype, int D, const cache_view& c, int heads_q, int n, const row_view& q,
                             const int32_t* length, const int32_t* count, bool causal, const row_view& o, float* lse,
                             void* ws, hipStream_t s) {
    const attn_plan p = plan_attn(dtype, D, c, heads_q, n);
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
    a.causal = causal;
    a.pieces = static_cast<uint32_t>(static_cast<int64_t>(c.batch) * c.heads * p.splits);
    a.spread = p.tile_rows != ROWS || a.pieces >= 128;
    if (dtype == 0 && D == 64) launch_attn<float, 64>(a, p, s);
    else if (dtype == 0) launch_attn<float, 128>(a, p, s);
    else if (D == 64) launch_attn<bf16_t, 64>(a, p, s);
    else launch_attn<bf16_t, 128>(a, p, s);
    return hipGetLastError();
}

}  // namespace vsa2
