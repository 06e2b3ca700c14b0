// Device-side parts of the attentions over the paged 8-bit cache: what a wave does with
// a page for its rows, and the two kernels' bodies (few rows, many rows), which
// attn_cache.hip, attn_cache_shared.hip and attn_cache_scored.hip launch.
#pragma once

#include <cfloat>

#include "common.hpp"

namespace vsa2 {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;

constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.44269504088896340f;
constexpr int TILE = 16;          // rows of a tile of tile_body
constexpr int NW = 4;             // waves of a workgroup of rows_body
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
    int samples;         // sequences that share a list (SHARED rows)
    uint32_t pieces;     // of all lists
    bool causal, spread;
};

// Whose rows a body works on and where they go: a list's own sequence, results written, or
// partial results where the list is in several pieces (WHOLE); the same, always partial
// results (OWN); all sequences that share the list, always partial results (SHARED).
enum rows_kind { WHOLE, OWN, SHARED };

// How rows see a list.  Plain: the positions below a limit.
struct plain_scores {
    static constexpr bool ON = false;
    struct row { int limit; };
};
// Scored: capped scores, a bias by distance, and two ranges of positions, [0, sinks) and [lo, hi).
// The options are the same for all rows of a call.
struct scored : score_options {
    static constexpr bool ON = true;
    struct row {
        int sinks, lo, hi;
        int at;          // the token's own position
        float slope;     // times log2 e
    };
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

// Zeros instead of fragments.
template <int N>
__device__ __forceinline__ void zeros_if(bool no, frag_bf16* f) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;
#pragma unroll
    for (int x = 0; x < N; ++x) {
        u32x4_t w = __builtin_bit_cast(u32x4_t, f[x].v);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = no ? 0u : w[i];
        f[x].v = __builtin_bit_cast(bf16x8_t, w);
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
template <rows_kind KIND>
__device__ __forceinline__ int row_limit(const attn_args& a, int b, int r) {
    if (r >= a.rows) return 0;
    int i = r / a.group, seq = b;
    if constexpr (KIND == SHARED) {
        seq = b * a.samples + i / a.n;
        i %= a.n;
    }
    int cnt = a.n;
    if (a.count) cnt = min(max(a.count[seq], 0), a.n);
    if (i >= cnt) return 0;
    const int64_t most = static_cast<int64_t>(a.c.max_pages) * CACHE_TOKENS;
    int64_t len = a.length[b];
    len = len < 0 ? 0 : (len > most ? most : len);
    if (KIND != SHARED && a.causal) len -= cnt - 1 - i;
    return static_cast<int>(len < 0 ? 0 : len);
}

// The same of a scored call; a row that sees nothing has sinks <= 0 and hi <= lo.
__device__ __forceinline__ scored::row scored_row(const attn_args& a, const scored& sc, int b, int h, int r) {
    scored::row w{0, 0, 0, 0, 0.f};
    const int limit = row_limit<WHOLE>(a, b, r);
    if (limit <= 0) return w;
    const int i = r / a.group;
    int cnt = a.n;
    if (a.count) cnt = min(max(a.count[b], 0), a.n);
    const int64_t most = static_cast<int64_t>(a.c.max_pages) * CACHE_TOKENS;
    int64_t len = a.length[b];
    len = len < 0 ? 0 : (len > most ? most : len);
    w.at = static_cast<int>(len - cnt + i);          // above -2^31: lengths are 0 at least
    w.hi = limit;
    w.sinks = min(sc.sink, limit);
    if (sc.window) w.lo = static_cast<int>(max(static_cast<int64_t>(0), static_cast<int64_t>(w.at) + 1 - sc.window));
    if (sc.span) {
        const int32_t* sp = sc.span + 2 * (static_cast<int64_t>(b) * a.n + i);
        w.lo = max(w.lo, sp[0]);
        w.hi = max(0, min(w.hi, sp[1]));
    }
    if (sc.slope) w.slope = sc.slope[h * a.group + (r - i * a.group)] * LOG2E;
    return w;
}
__device__ __forceinline__ bool sees_nothing(const plain_scores::row& w) { return w.limit == 0; }
__device__ __forceinline__ bool sees_nothing(const scored::row& w) { return w.sinks <= 0 && w.hi <= w.lo; }

// Of four positions from `first` on, a bit for each that the row sees.
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 4 ? 15u : (n <= 0 ? 0u : (1u << n) - 1); }
__device__ __forceinline__ uint32_t seen_bits(const scored::row& w, int first) {
    return first_bits(w.sinks - first) | (first_bits(w.hi - first) & ~first_bits(w.lo - first));
}
// 0xff for each of four bits.
__device__ __forceinline__ uint32_t bytes_of(uint32_t bits) { return ((bits * 0x00204081u) & 0x01010101u) * 0xffu; }
// The or over the 16 lanes of a group.
__device__ __forceinline__ uint32_t lanes_or(uint32_t x) {
    x |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xB1, 0xF, 0xF, false));
    x |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x4E, 0xF, 0xF, false));
    x |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x141, 0xF, 0xF, false));
    x |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x140, 0xF, 0xF, false));
    return x;
}

// Of the 32 positions that one half of a wave's lanes holds of a page (first + 8 x + i, x below 8, i
// below 4), a bit for each that the row sees, and that some row of the half's lanes sees.
__device__ __forceinline__ uint32_t half_bits(const scored::row& w, int first) {
    uint32_t bits = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) bits |= seen_bits(w, first + 8 * x) << (4 * x);
    return bits;
}
__device__ __forceinline__ uint32_t half_union(uint32_t bits) {
    bits = lanes_or(bits);
    return bits | static_cast<uint32_t>(__shfl_xor(static_cast<int>(bits), 16, 64));
}

// What the rows of a tile see together, the same in every lane: the ends of all their
// ranges, for the pages that are visited, and what every row that sees something
// sees, for those that need no mask.
struct scored_ends {
    int sinks, lo, hi;               // union's ends
    int all_sinks, all_lo, all_hi;   // seen by all: [0, all_sinks) and [all_lo, all_hi)

    __device__ __forceinline__ void none() {
        sinks = hi = 0;
        lo = all_sinks = all_lo = all_hi = INT32_MAX;
        all_lo = INT32_MIN;
    }
    __device__ __forceinline__ void add(const scored::row& w) {
        if (sees_nothing(w)) return;
        const bool range = w.hi > w.lo;
        sinks = max(sinks, w.sinks);
        all_sinks = min(all_sinks, w.sinks);
        lo = range ? min(lo, w.lo) : lo;
        hi = range ? max(hi, w.hi) : hi;
        all_lo = range ? max(all_lo, w.lo) : INT32_MAX;
        all_hi = range ? min(all_hi, w.hi) : 0;
    }
    __device__ __forceinline__ void join(const scored_ends& o) {
        sinks = max(sinks, o.sinks);
        lo = min(lo, o.lo);
        hi = max(hi, o.hi);
        all_sinks = min(all_sinks, o.all_sinks);
        all_lo = max(all_lo, o.all_lo);
        all_hi = min(all_hi, o.all_hi);
    }
    // over LANES neighbouring lanes, then made uniform
    template <int LANES>
    __device__ __forceinline__ void reduce() {
#pragma unroll
        for (int m = LANES / 2; m; m >>= 1) {
            const scored_ends o{__shfl_xor(sinks, m, 64),     __shfl_xor(lo, m, 64),     __shfl_xor(hi, m, 64),
                                __shfl_xor(all_sinks, m, 64), __shfl_xor(all_lo, m, 64), __shfl_xor(all_hi, m, 64)};
            join(o);
        }
        sinks = __builtin_amdgcn_readfirstlane(sinks);
        lo = __builtin_amdgcn_readfirstlane(lo);
        hi = __builtin_amdgcn_readfirstlane(hi);
        all_sinks = __builtin_amdgcn_readfirstlane(all_sinks);
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }
    // pages from the list's start, then pages [second, second + more)
    __device__ __forceinline__ int front() const { return (sinks + CACHE_TOKENS - 1) / CACHE_TOKENS; }
    __device__ __forceinline__ int second() const { return max(lo / CACHE_TOKENS, front()); }
    __device__ __forceinline__ int more() const { return max(0, (hi + CACHE_TOKENS - 1) / CACHE_TOKENS - second()); }
    __device__ __forceinline__ bool whole(int page) const {
        const int first = page * CACHE_TOKENS, end = first + CACHE_TOKENS;
        return end <= all_sinks || (first >= all_lo && end <= all_hi);
    }
    __device__ __forceinline__ bool sees(int page) const {
        const int first = page * CACHE_TOKENS;
        return first < sinks || (first < hi && first + CACHE_TOKENS > lo);
    }
};

// The options' part of a score, in base 2: log2 e (cap tanh(x / cap) - slope |at - position|) of
// x = s * scale.
//
// tanh(y) = 1 - 2 / (e^2y + 1), or, below 0.5, the odd polynomial y + a y^3 + b y^5 + c y^7 that is
// nearest to it there (by linear programming over 3,001 points; off by 2^-22.3 at most, of a score
// by 2^-22.3 of the cap and by 2^-19.9 of itself): s times a polynomial of s^2.  Where all of a
// wave's scores that some row sees are small only that is worked out, the bias added by the same
// instructions.  Elsewhere the first serves all of the wave's scores up to caps of 2^8, off by
// 2^-22 of the cap (2^-14: a sixty-fourth of the result's rounding), and a score takes the one that
// is its own above, where small ones would lose bits (0.08 of a score of 1 at a cap of 2^20); that
// for all caps took 238 us of the capped frame below instead of 202.  fp32 queries take scores
// below 0.4 by the series instead, the others as above: the difference would cost them bits (cap
// 50: 2^-17 of the weights).  A page behind all rows' own positions, or more than a page before
// them, has a bias that is linear in the position; nearer ones take distances as whole numbers, so
// that an own position has no bias at all.  1,792 tokens over 10,752, 12 heads of 128: 148 us
// without options (plain attention 144), 165 with a bias, 185 with a cap that the polynomial
// serves, 203 with one that it does not, 193 with the first cap and a bias (by the polynomial the
// capped frame of attn_cache_scored.hip went from 222 to 212 us).
template <bool EXACT>
struct score_form {
    float scale, cap, rate;      // scale times log2 e, cap times log2 e, exponent of a score
    float cut;                   // scale / cap
    float small;                 // scores below this take the polynomial
    float c1, c2, c3;            // its factors of s^2, s^4, s^6, times scale (caps are 2^-20 to 2^20: all finite)
    bool capped, sloped;
    __device__ __forceinline__ score_form(const scored& sc, int D) {
        const float root = 1.f / sqrtf(static_cast<float>(D));
        capped = sc.cap > 0.f;
        sloped = sc.slope != nullptr;
        scale = root * LOG2E;
        cap = sc.cap * LOG2E;
        cut = capped ? root / sc.cap : 0.f;
        rate = 2.f * LOG2E * cut;
        small = 0.5f / cut;
        const float u = cut * cut;
        c1 = scale * u * -0.33326461f;
        c2 = scale * u * u * 0.13185862f;
        c3 = scale * u * u * u * -0.0442293f;
    }
    // the polynomial, and the bias
    __device__ __forceinline__ float small_of(float s, float bias) const {
        const float u = s * s;
        return fmaf(s, fmaf(u, fmaf(u, fmaf(u, c3, c2), c1), scale), bias);
    }
    __device__ __forceinline__ float capped_of(float s) const {
        const float e = fast_exp2(EXACT ? fabsf(s) * rate : s * rate);
        if constexpr (!EXACT) return fmaf(-2.f * cap, __builtin_amdgcn_rcpf(e + 1.f), cap);
        const float y = s * cut, u = y * y;
        float p = fmaf(u, 21844.f / 6081075.f, -1382.f / 155925.f);
        p = fmaf(u, p, 62.f / 2835.f);
        p = fmaf(u, p, -17.f / 315.f);
        p = fmaf(u, p, 2.f / 15.f);
        p = fmaf(u, p, -1.f / 3.f);
        const float near = cap * fmaf(y * u, p, y);
        const float far = copysignf(cap * fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f), s);
        return fabsf(y) < 0.4f ? near : far;         // a NaN stays one
    }
    // The scores s[t][i], t below TILES, of the page at `first`, at positions here + place(t, i);
    // masks: those without their bit in `bits` (N t + i) may be anything, and choose no form for the others;
    // returns what the results are still to be multiplied with (the same for all).
    template <int TILES, int N, typename V, typename P>
    __device__ __forceinline__ float apply(V* s, const scored::row& w, int first, int here, bool masks, uint32_t bits,
                                           P place) const {
        if (!capped && !sloped) return scale;
        const float away = static_cast<float>(w.at - here);
        float a = 0.f, slant = 0.f;             // a linear bias: a + slant * place
        bool linear = true;
        if (sloped) {
            // a page away at least: a, which the last terms take back, is twice the bias there at most
            const bool before = w.at >= first + 2 * CACHE_TOKENS - 1, behind = w.at <= first;
            linear = __ballot(!before && !behind) == 0;
            slant = behind ? -w.slope : w.slope;
            a = -slant * away;
        }
        bool poly = !capped;
        if (capped) {
            float most = 0.f;
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < N; i += 2) most = fmaxf(fmaxf(most, fabsf(s[t][i])), fabsf(s[t][i + 1]));
            if (masks) {
                most = 0.f;
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        int seen = static_cast<int>(bits << (31 - (N * t + i))) >> 31;
                        asm("" : "+v"(seen));          // kept in a vector register: as many masks would not fit the scalar ones
                        most = fmaxf(most, fabsf(__uint_as_float(__float_as_uint(s[t][i]) & static_cast<uint32_t>(seen))));
                    }
            }
            poly = !EXACT && __ballot(most >= small) == 0;          // (a NaN goes through either)
        }
        if (poly && linear) {
            if (capped) {
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int i = 0; i < N; ++i) s[t][i] = small_of(s[t][i], a);
            } else {
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int i = 0; i < N; ++i) s[t][i] = fmaf(s[t][i], scale, a);
            }
            if (!sloped) return 1.f;
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < N; ++i) s[t][i] = fmaf(slant, static_cast<float>(place(t, i)), s[t][i]);
            return 1.f;
        }
        if (!EXACT && cap > 256.f * LOG2E) {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float far = capped_of(s[t][i]);
                    s[t][i] = fabsf(s[t][i]) < small ? small_of(s[t][i], 0.f) : far;         // a NaN stays one
                }
        } else {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int i = 0; i < N; ++i) s[t][i] = capped ? capped_of(s[t][i]) : s[t][i] * scale;
        }
        if (!sloped) return 1.f;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < N; ++i)
                s[t][i] = fmaf(-w.slope, fabsf(away - static_cast<float>(place(t, i))), s[t][i]);
        return 1.f;
    }
};
// Plain scores: nothing but the scale, which the softmax applies.
struct plain_form {
    float scale;
    __device__ __forceinline__ plain_form(const plain_scores&, int D) : scale(LOG2E / sqrtf(static_cast<float>(D))) {}
};
template <typename T, class SC> struct form_of { using type = plain_form; };
template <typename T> struct form_of<T, scored> { using type = score_form<sizeof(T) == 4>; };
template <typename T, class SC> using form_of_t = typename form_of<T, SC>::type;

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
template <bool GAP>
struct page_walk {
    const int32_t* table;
    int at, hi, pages;     // next entries to fetch; pages of the pool
    int ids, base;         // fetched entries (one per lane), their first position
    int front = 0, gap = 0;     // GAP: `gap` pages left out behind the first `front`
    uint64_t left;         // of those, still to visit

    __device__ __forceinline__ page_walk(const int32_t* t, int lo, int hi_, int n)
        : table(t), at(lo), hi(hi_), pages(n), ids(-1), base(lo), left(0) {}
    __device__ __forceinline__ int slot(int x) const { return GAP && x >= front ? x + gap : x; }
    // `mine`: which of 64 entries in a row the caller visits
    __device__ __forceinline__ void fetch(uint64_t mine) {
        const int x = at + lane_id();
        start(x < hi ? table[slot(x)] : -1, mine);
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
        pos = slot(base + bit);
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
__device__ __forceinline__ uint32_t piece_of(const attn_args& a, uint32_t block, uint32_t blocks, int& tile) {
    if (!a.spread) {
        const uint32_t item = static_cast<uint32_t>(xcd_item(block, blocks));
        tile = static_cast<int>(item % a.tiles);
        return item / a.tiles;
    }
    const uint32_t turn = block >> 3, t = turn / a.tiles;
    tile = static_cast<int>(turn - t * a.tiles);
    return t * 8 + (block & 7);
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

// One page for XT tiles, decoded once for all of them.  masks: some row's limit, or the list's
// end, may lie inside it; known where this is compiled for plain scores (a loop without masks
// and one with them), at run time for others, whose masked pages come first and last: two loops
// inside one cost the rows' registers a second time.
template <typename T, int D, int XT, class SC>
__device__ __forceinline__ void page_step(const page_data<D>& pd, const char* page, int pos,
                                          const typename SC::row (&row)[XT], int lim_max, bool masks,
                                          const frag_bf16 (&qf)[XT][D / 32][terms_of<T>], const form_of_t<T, SC>& form,
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
    float scale = form.scale;
    uint32_t vw[4] = {pd.ve.x, pd.ve.y, pd.ve.z, pd.ve.w};
    uint4 vr[D / 16];
#pragma unroll
    for (int c = 0; c < D / 16; ++c) vr[c] = pd.v[c];
    weight_frag_t<T> pf[XT][2][NT];
    // a quarter of the lane's tokens' powers, of those below lim_max
    const int at = lane_id() & 3;
    const uint32_t four = at & 2 ? (at & 1 ? vw[3] : vw[2]) : (at & 1 ? vw[1] : vw[0]);
    uint32_t marked = ~0u;
    uint32_t bits[XT] = {}, together = 0;      // scored, masked: what this lane's row, and some row, sees of its tokens
    if (SC::ON && masks) {
        if constexpr (SC::ON) {
#pragma unroll
            for (int x = 0; x < XT; ++x) {
#pragma unroll
                for (int t = 0; t < 4; ++t) bits[x] |= seen_bits(row[x], pos + 16 * t + 4 * g) << (4 * t);
                together |= bits[x];
            }
        }
        together = lanes_or(together);
        marked = bytes_of((together >> (4 * at)) & 15u);
    } else if (masks) {
        marked = first_bytes(lim_max - (pos + 16 * at + 4 * g));
    }
    float mx[XT];
    const bool news = NT == 1 && seen.news(four, marked);
    bool far = false;
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        if constexpr (SC::ON) {
            scale = form.template apply<4, 4>(s[x], row[x], pos, pos + 4 * g, masks, bits[x], [](int t, int i) { return 16 * t + i; });
        }
        if (masks) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (SC::ON) {
                        if (!((bits[x] >> (4 * t + i)) & 1u)) s[x][t][i] = -INFINITY;
                    } else {
                        if (pos + 16 * t + 4 * g + i >= row[x].limit) s[x][t][i] = -INFINITY;
                    }
                }
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
    if (SC::ON && masks) {
        // what no row sees may hold any power: one that a weight of 0 leaves 0
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t real = bytes_of((together >> (4 * t)) & 15u);
            vw[t] = (vw[t] & real) | (static_cast<uint32_t>(seen.most) * 0x01010101u & ~real);
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
                p[t][i] = !SC::ON && masks && e == 0.f ? 0.f : e * (NT == 1 ? seen.scaled(byte) : power_of(byte));
            }
        w.l = fmaf(sum, w.down, w.l);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const float z[8] = {p[2 * y][0], p[2 * y][1], p[2 * y][2], p[2 * y][3],
                                p[2 * y + 1][0], p[2 * y + 1][1], p[2 * y + 1][2], p[2 * y + 1][3]};
            split_weights<NT>(pf[x][y], z);
        }
    }
    uint32_t keep[4] = {}, any = 0;
    if (masks) {
        // Codes past every row's limit are whatever the page held: taken as
        // zeros.  A NaN below it, which some rows see and others do not, is
        // taken out of the product, too.
#pragma unroll
        for (int t = 0; t < 4; ++t)
            keep[t] = SC::ON ? bytes_of((together >> (4 * t)) & 15u) : first_bytes(lim_max - (pos + 16 * t + 4 * g));
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
    if (masks) {
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
                f32x4_t hit = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if constexpr (SC::ON) {
                    uint32_t one[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) one[t] = bytes_of((bits[x] >> (4 * t)) & 15u) & ONE_E4M3;
                    hit = mma16(decode8(nan[0], nan[1], 1.f), decode8(one[0], one[1], 1.f), hit);
                    hit = mma16(decode8(nan[2], nan[3], 1.f), decode8(one[2], one[3], 1.f), hit);
                } else {
                    const int here = row[x].limit - (pos + 4 * g);
                    hit = mma16(decode8(nan[0], nan[1], 1.f), shown8(here, here - 16), hit);
                    hit = mma16(decode8(nan[2], nan[3], 1.f), shown8(here - 32, here - 48), hit);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    st[x].o[c][i] += nan_if(hit[i]);
            }
        }
    }
}

// Element offset of row r (query head and token of KV head h) in q or o.
template <rows_kind KIND = WHOLE>
__device__ __forceinline__ int64_t row_offset(const row_view& v, const attn_args& a, int b, int h, int r) {
    int i = r / a.group;
    const int hg = r - i * a.group;
    if constexpr (KIND == SHARED) {
        b = b * a.samples + i / a.n;
        i %= a.n;
    }
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
template <int D, int WAVES, int XT>
struct tile_lds {
    float so[WAVES][XT * TILE][D + 4];
    float sml[WAVES][XT * TILE][2];
};
template <typename T, int D, int WAVES, int XT, rows_kind KIND, class SC>
__device__ __forceinline__ void tile_body(const attn_args& a, const SC& sc, uint32_t block, uint32_t blocks,
                                          tile_lds<D, WAVES, XT>& lds) {
    constexpr int NT = terms_of<T>, TR = XT * TILE;
    auto& so = lds.so;
    auto& sml = lds.sml;
    const int lane = lane_id(), wave = wave_id(), g = lane >> 4, col = lane & 15;
    int tile;
    const uint32_t item = piece_of(a, block, blocks, tile);
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
    const int early = !SC::ON && a.splits == 1 && lane < a.c.max_pages ? list[lane] : -1;
    // rows that see nothing compute with queries of zeros, which leave the others alone, and drop it at the end
    typename SC::row row[XT];
    int lim_max = 0, lim_min = 0, pages;
    scored_ends ends;
    if constexpr (SC::ON) {
        ends.none();
#pragma unroll
        for (int x = 0; x < XT; ++x) {
            row[x] = scored_row(a, sc, b, h, tile * TR + x * TILE + col);
            ends.add(row[x]);
        }
        ends.template reduce<16>();
        pages = ends.front() + ends.more();
    } else {
        int most = 0, least = INT32_MAX;
#pragma unroll
        for (int x = 0; x < XT; ++x) {
            row[x].limit = row_limit<KIND>(a, b, tile * TR + x * TILE + col);
            most = max(most, row[x].limit);
            least = row[x].limit > 0 ? min(least, row[x].limit) : least;
        }
        lim_max = __builtin_amdgcn_readfirstlane(lanes_max(most));
        lim_min = __builtin_amdgcn_readfirstlane(lanes_min(least));
        pages = (lim_max + CACHE_TOKENS - 1) / CACHE_TOKENS;
    }
    const int lo = static_cast<int>(static_cast<int64_t>(pages) * split / a.splits);
    const int hi = static_cast<int>(static_cast<int64_t>(pages) * (split + 1) / a.splits);
    page_walk<SC::ON> walk(list, lo, hi, a.c.pages);
    if constexpr (SC::ON) {
        walk.front = ends.front();
        walk.gap = ends.second() - ends.front();
        if (lo < hi) walk.fetch(mine);
    } else {
        if (a.splits == 1) walk.start(early, mine);
        else if (lo < hi) walk.fetch(mine);
    }

    frag_bf16 qf[XT][D / 32][NT];
    tile_state<T, D> st[XT];
    powers_seen seen;
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        const int r = tile * TR + x * TILE + col;
        const T* q = static_cast<const T*>(a.q.ptr) + (r < a.rows ? row_offset<KIND>(a.q, a, b, h, r) : 0);
        // (read before it is known, so that lengths and queries are waited for together)
        const bool dead = sees_nothing(row[x]);
#pragma unroll
        for (int u = 0; u < D / 32; ++u) {
            float y[8] = {};
            if (r < a.rows) {
                const T* e = q + (u / 2) * 64 + g * 16 + (u & 1) * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = to_f32(e[i]);
            }
            split_frag<NT>(qf[x][u], y);
            zeros_if<NT>(dead, qf[x][u]);
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) st[x].o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const form_of_t<T, SC> form(sc, D);
    int pg, id;
    bool more = walk.next(pg, id, mine);
    const auto page = [&]() { return a.c.pool + (static_cast<int64_t>(id) * a.c.heads + h) * cache_page_bytes(D); };
    const auto whole = [&]() { return more && (pg + 1) * CACHE_TOKENS <= lim_min; };
    if constexpr (SC::ON) {
        for (; more; more = walk.next(pg, id, mine)) {
            page_data<D> x;
            load_page<D>(x, page());
            page_step<T, D, XT, SC>(x, page(), pg * CACHE_TOKENS, row, lim_max, !ends.whole(pg), qf, form, st, seen);
        }
    } else {
        for (; whole(); more = walk.next(pg, id, mine)) {
            page_data<D> x;
            load_page<D>(x, page());
            page_step<T, D, XT, SC>(x, nullptr, 0, row, lim_max, false, qf, form, st, seen);
        }
        for (; more; more = walk.next(pg, id, mine)) {
            page_data<D> x;
            load_page<D>(x, page());
            page_step<T, D, XT, SC>(x, page(), pg * CACHE_TOKENS, row, lim_max, true, qf, form, st, seen);
        }
    }
#pragma unroll
    for (int x = 0; x < XT; ++x) {
        float l = st[x].w.l;
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        const bool dead = sees_nothing(row[x]);
        const int at = x * TILE + col;
        const float back = seen.back(st[x].w);
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            *reinterpret_cast<f32x4_t*>(&so[wave][at][16 * c + 4 * g]) =
                dead ? f32x4_t{0.f, 0.f, 0.f, 0.f} : st[x].o[c] * back;
        if (g == 0) {
            sml[wave][at][0] = dead ? -INFINITY : st[x].w.m();
            sml[wave][at][1] = dead ? 0.f : l;
        }
    }
    __syncthreads();
    // join the waves: a thread takes 4 elements of a row
    for (int at = threadIdx.x; at < TR * (D / 4); at += 64 * WAVES) {
        const int tr = at / (D / 4), d0 = at % (D / 4) * 4, rr = tile * TR + tr;
        if (rr >= a.rows) continue;
        float m = sml[0][tr][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sml[w][tr][0]);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f, o[4] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = fast_exp2(sml[w][tr][0] - base);
            const float4 y = *reinterpret_cast<const float4*>(&so[w][tr][d0]);
            l += f * sml[w][tr][1];
            o[0] += f * y.x;
            o[1] += f * y.y;
            o[2] += f * y.z;
            o[3] += f * y.w;
        }
        if (KIND != WHOLE || a.splits > 1) {
            float* part = a.part + ((static_cast<int64_t>(bh) * a.tiles + tile) * a.splits + split) * (TR * (D + 2));
            store4(part + tr * D + d0, o);
            if (d0 == 0) {
                part[TR * D + 2 * tr] = m;
                part[TR * D + 2 * tr + 1] = l;
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
    bool wide = false;          // a lane's token of each page more than 2^7 below E (or past all limits)
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

// One page in LDS for a wave's rows, where (plain scores) some row's limit, or the list's end,
// may lie inside it, or (others) `masks` says so.
template <typename T, int D, class SC>
__device__ __forceinline__ void rows_step(const char* kp, const char* vp, const float (*page_power)[2][64], int first,
                                          const typename SC::row& row, int wmax, bool masks,
                                          const frag_bf16 (&qf)[D / 32][2][terms_of<T>], const form_of_t<T, SC>& form,
                                          powers_seen& seen, rows_state<T, D>& st) {
    const float (*power)[64] = *page_power;
    float scale = form.scale;
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
    uint32_t bits = 0, together = 0;       // scored: what this lane's row, and some row, sees of its 32 tokens
    if constexpr (SC::ON) {
        if (masks) {
            bits = half_bits(row, first + 4 * h2);
            together = half_union(bits);
        }
        scale = form.template apply<2, 16>(s, row, first, first + 4 * h2, masks, bits,
                                           [](int t, int i) { return t * 32 + 8 * (i / 4) + i % 4; });
        if (masks) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = (bits >> (16 * t + i)) & 1u ? s[t][i] : -INFINITY;
        }
    } else {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (first + t * 32 + 8 * (i / 4) + 4 * h2 + i % 4 >= row.limit) s[t][i] = -INFINITY;
    }
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
                // a masked place's power may be anything (scored: not what is in LDS)
                y[4 * x + i] = !SC::ON && y[4 * x + i] == 0.f ? 0.f : y[4 * x + i] * pv[i];
            }
        }
        split_weights<NT>(pf[t], y);
    }
    st.w.l = fmaf(sum, st.w.down, st.w.l);
    uint32_t keep[4][2], any = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x)
            keep[t][x] = SC::ON ? bytes_of((together >> (8 * t + 4 * x)) & 15u)
                                : first_bytes(wmax - (first + 16 * t + 8 * x + 4 * h2));
    // as in page_step: stale codes are zeros, a NaN goes to the rows that see it; scored: only
    // where there is a NaN, the weight of the others is 0
    bool odd = !SC::ON;
    if (SC::ON && masks) {
        uint32_t nans = 0;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint4 v = *reinterpret_cast<const uint4*>(vp + c * 2048 + 512 * x);
                nans |= nan_bytes(v.x) | nan_bytes(v.y) | nan_bytes(v.z) | nan_bytes(v.w);
            }
        odd = __ballot(nans != 0) != 0;
    }
#pragma unroll
    for (int c = 0; c < VC; ++c) {
        const uint4 va = *reinterpret_cast<const uint4*>(vp + c * 2048);
        const uint4 vb = *reinterpret_cast<const uint4*>(vp + c * 2048 + 512);
        uint32_t w[4][2] = {{va.x, vb.x}, {va.y, vb.y}, {va.z, vb.z}, {va.w, vb.w}};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (odd) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    w[t][x] &= keep[t][x];
                    const uint32_t nan = nan_bytes(w[t][x]);
                    w[t][x] &= ~nan;
                    any |= nan;
                }
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
            const frag_bf16 nan =
                decode8(nan_bytes(w[t][0] & keep[t][0]) & ONE_E4M3, nan_bytes(w[t][1] & keep[t][1]) & ONE_E4M3, 1.f);
            if constexpr (SC::ON) {
                mma(hit, nan, decode8(bytes_of((bits >> (8 * t)) & 15u) & ONE_E4M3,
                                      bytes_of((bits >> (8 * t + 4)) & 15u) & ONE_E4M3, 1.f));
            } else {
                const int here = row.limit - (first + 16 * t + 4 * h2);
                mma(hit, nan, shown8(here, here - 8));
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            st.o[c][i] += nan_if(hit[i]);
    }
}

// The two pages of a stage together, no limit inside either.
template <typename T, int D, class SC>
__device__ __forceinline__ void rows_pair(const char* lds, int kbase, int vbase, const float (*power)[2][64],
                                          const int (&pages)[STAGE], const typename SC::row& row,
                                          const frag_bf16 (&qf)[D / 32][2][terms_of<T>], const form_of_t<T, SC>& form,
                                          powers_seen& seen, rows_state<T, D>& st) {
    float scale = form.scale;
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
    if constexpr (SC::ON) {
#pragma unroll
        for (int x = 0; x < STAGE; ++x) {
            const int first = pages[x] * CACHE_TOKENS;
            scale = form.template apply<2, 16>(s + 2 * x, row, first, first + 4 * h2, false, 0,
                                       [](int t, int i) { return t * 32 + 8 * (i / 4) + i % 4; });
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

template <int D>
struct rows_lds {
    __attribute__((aligned(1024))) char codes[2][STAGE][128 * D];
    __attribute__((aligned(16))) float power[NW][STAGE][2][64];
    int ends[NW][8];
};
template <typename T, int D, rows_kind KIND, class SC>
__device__ __forceinline__ void rows_body(const attn_args& a, const SC& sc, uint32_t block, uint32_t blocks, rows_lds<D>& lds) {
    constexpr int NT = terms_of<T>, KC = D / 32, VC = D / 32;
    auto& codes = lds.codes;
    auto& power = lds.power;
    const int lane = lane_id(), wave = wave_id(), h2 = lane >> 5, col = lane & 31;
    int tile;
    const uint32_t item = piece_of(a, block, blocks, tile);
    if (item >= a.pieces) return;
    const int split = static_cast<int>(item % a.splits);
    const uint32_t bh = item / a.splits;
    const int b = static_cast<int>(bh / a.c.heads), h = static_cast<int>(bh % a.c.heads);
    const int r = tile * ROWS + wave * 32 + col;
    typename SC::row row;
    int wmax = 0, full = 0, pages;
    scored_ends wave_ends, ends;          // of the wave's rows and the workgroup's
    if constexpr (SC::ON) {
        row = scored_row(a, sc, b, h, r);
        wave_ends.none();
        wave_ends.add(row);
        wave_ends.template reduce<32>();
        if (lane == 0) {
            int* e = lds.ends[wave];
            e[0] = wave_ends.sinks, e[1] = wave_ends.lo, e[2] = wave_ends.hi;
            e[3] = wave_ends.all_sinks, e[4] = wave_ends.all_lo, e[5] = wave_ends.all_hi;
        }
        __syncthreads();
        ends.none();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int* e = lds.ends[w];
            ends.join(scored_ends{e[0], e[1], e[2], e[3], e[4], e[5]});
        }
        ends.template reduce<1>();
        pages = ends.front() + ends.more();
    } else {
        // the rows' limits: the wave's largest, the workgroup's largest and (of rows that see something,
        // the others drop what they compute at the end) smallest
        row.limit = row_limit<KIND>(a, b, r);
        int wmin = row.limit > 0 ? row.limit : INT32_MAX;
        wmax = row.limit;
#pragma unroll
        for (int m = 16; m; m >>= 1) {
            wmin = min(wmin, __shfl_xor(wmin, m, 64));
            wmax = max(wmax, __shfl_xor(wmax, m, 64));
        }
        wmax = __builtin_amdgcn_readfirstlane(wmax);
        if (lane == 0) {
            lds.ends[wave][0] = wmin;
            lds.ends[wave][1] = wmax;
        }
        __syncthreads();
        int all = 0;
        full = INT32_MAX;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            full = min(full, lds.ends[w][0]);
            all = max(all, lds.ends[w][1]);
        }
        all = __builtin_amdgcn_readfirstlane(all);
        full = __builtin_amdgcn_readfirstlane(full) / CACHE_TOKENS;     // pages before this one need no mask
        pages = (all + CACHE_TOKENS - 1) / CACHE_TOKENS;
    }
    const int lo = static_cast<int>(static_cast<int64_t>(pages) * split / a.splits);
    const int hi = static_cast<int>(static_cast<int64_t>(pages) * (split + 1) / a.splits);

    frag_bf16 qf[KC][2][NT];
    const bool dead = sees_nothing(row);       // queries of zeros, which leave the others alone
    const T* q = static_cast<const T*>(a.q.ptr) + (r < a.rows ? row_offset<KIND>(a.q, a, b, h, r) : 0);
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
            zeros_if<NT>(dead, qf[w][z]);
        }
    rows_state<T, D> st;
    powers_seen seen;
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[c][i] = 0.f;
    const form_of_t<T, SC> form(sc, D);
    const int kbase = (col >> 4) * (D / 64) * 1024 + h2 * 256 + (col & 15) * 16;
    const int vbase = 64 * D + (col >> 4) * 1024 + h2 * 256 + (col & 15) * 16;
    // in-page places of this lane's token's two powers
    const int ke_at = 128 * D + (lane & 15) * 4 + (lane >> 4);
    const int ve_at = 128 * D + 64 + ((lane >> 2) & 3) * 16 + (lane >> 4) * 4 + (lane & 3);

    page_walk<SC::ON> walk(list_of(a, b, h), lo, hi, a.c.pages);
    if constexpr (SC::ON) {
        walk.front = ends.front();
        walk.gap = ends.second() - ends.front();
    }
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
        uint32_t mine[STAGE];            // scored: is the lane's token seen by some row of the wave (all ones)?
        if constexpr (SC::ON) {
            // what lies between the rows' ranges may never have been written
#pragma unroll
            for (int x = 0; x < STAGE; ++x) {
                mine[x] = x < have && wave_ends.whole(pos[x]) ? ~0u : 0u;
                if (!mine[x] && x < have && wave_ends.sees(pos[x])) {
                    const uint32_t here = half_union(half_bits(row, pos[x] * CACHE_TOKENS + 4 * h2));
                    const uint32_t there = static_cast<uint32_t>(__shfl_xor(static_cast<int>(here), 32, 64));
                    mine[x] = 0u - ((((lane >> 2) & 1) == h2 ? here : there) >> (4 * (lane >> 3) + (lane & 3)) & 1u);
                }
            }
        }
        if constexpr (NT == 1) {
            uint32_t marked = 0;
#pragma unroll
            for (int x = 0; x < STAGE; ++x) {
                if constexpr (SC::ON) marked |= (mine[x] & ve[x]) << (8 * x);
                else {
                    // past the wave's limits whatever the page holds: a power of 0, as on a page of zeros
                    if (x >= have || pos[x] * CACHE_TOKENS + lane >= wmax) ve[x] = 0;
                    marked |= static_cast<uint32_t>(ve[x]) << (8 * x);
                }
            }
            seen.look(marked);
        }
#pragma unroll
        for (int x = 0; x < STAGE; ++x) {
            power[wave][x][0][lane] = power_of(ke[x]);
            power[wave][x][1][lane] = NT == 1 ? seen.scaled(seen.raised(ve[x])) : power_of(ve[x]);
            if (SC::ON && !mine[x]) power[wave][x][1][lane] = 1.f;      // any that a weight of 0 leaves 0
            at[x] = pos[x];
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        wg_barrier();
        const int n = have;
        request(buf ^ 1);
        return n;
    };
    if constexpr (!SC::ON) {
        while (have == STAGE && pos[STAGE - 1] < full) {
            turn();
            // (a wave without rows: shared lists' last tile has few)
            if (KIND != SHARED || wmax > 0)
                rows_pair<T, D, SC>(codes[buf][0], kbase, vbase, power[wave], at, row, qf, form, seen, st);
            buf ^= 1;
        }
    }
    while (have > 0) {
        int n = turn();
        if (SC::ON && n == STAGE && wave_ends.whole(at[0]) && wave_ends.whole(at[STAGE - 1])) {
            rows_pair<T, D, SC>(codes[buf][0], kbase, vbase, power[wave], at, row, qf, form, seen, st);
            n = 0;
        }
#pragma unroll 1
        for (int x = 0; x < n; ++x) {
            const int pg = x ? at[STAGE - 1] : at[0], first = pg * CACHE_TOKENS;
            if (SC::ON ? wave_ends.sees(pg) : first < wmax)
                rows_step<T, D, SC>(codes[buf][x] + kbase, codes[buf][x] + vbase, &power[wave][x], first, row, wmax,
                                    SC::ON && !wave_ends.whole(pg), qf, form, seen, st);
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
    if (dead) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    }
    const float base = m == -INFINITY ? 0.f : m;
    if (r >= a.rows) return;
    if (KIND != WHOLE || a.splits > 1) {
        float* part = a.part + ((static_cast<int64_t>(bh) * a.tiles + tile) * a.splits + split) * (ROWS * (D + 2));
        const int tr = wave * 32 + col;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float x[4] = {o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]};
                store4(part + tr * D + c * 32 + 2 * i + 4 * h2, x);
            }
        if (h2 == 0) {
            part[ROWS * D + 2 * tr] = m;
            part[ROWS * D + 2 * tr + 1] = l;
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
static __global__ __launch_bounds__(SLICES > 8 ? 32 * SLICES : 256) void attn_cache_join_kernel(attn_args a, int tile_rows) {
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
// The rules, with c.max_pages as the longest list a row may see.
attn_plan plan_attn(int dtype, int D, const cache_view& c, int heads_q, int n);
// The arguments of a call in a plan's pieces.
attn_args plan_args(const attn_plan& p, const cache_view& c, int heads_q, int n, const row_view& q, const int32_t* length,
                    const int32_t* count, bool causal, const row_view& o, float* lse, void* ws);

// Launches a plan: GO has the kernels around the two bodies.
template <typename T, int D, class GO>
void launch_attn(const attn_args& a, const attn_plan& p, hipStream_t s, const GO& go) {
    const int64_t items = static_cast<int64_t>(a.c.batch) * a.c.heads * p.tiles;
    const int64_t pieces = a.spread ? (static_cast<int64_t>(a.pieces) + 7) / 8 * 8 : a.pieces;
    const dim3 grid(static_cast<unsigned>(pieces * p.tiles)), block(64 * p.waves);
    if (p.tile_rows == ROWS) go.template rows<T, D>(grid, block, s, a);
    else if (p.tile_rows == TILE) {
        if (p.waves == 8) go.template tiles<T, D, 8, 1>(grid, block, s, a);
        else go.template tiles<T, D, 4, 1>(grid, block, s, a);
    } else if constexpr (two_tiles<T, D>) {
        if (p.waves == 8) go.template tiles<T, D, 8, 2>(grid, block, s, a);
        else go.template tiles<T, D, 4, 2>(grid, block, s, a);
    }
    const auto rows_of = [&](int per_wg) { return dim3(static_cast<unsigned>(items * (p.tile_rows / per_wg))); };
    if (p.splits > 32)
        hipLaunchKernelGGL((attn_cache_join_kernel<T, D, 32>), rows_of(1), dim3(1024), 0, s, a, p.tile_rows);
    else if (p.splits > 8)
        hipLaunchKernelGGL((attn_cache_join_kernel<T, D, 8>), rows_of(1), dim3(256), 0, s, a, p.tile_rows);
    else if (p.splits > 1)
        hipLaunchKernelGGL((attn_cache_join_kernel<T, D, 1>), rows_of(8), dim3(256), 0, s, a, p.tile_rows);
}

}  // namespace vsa2
