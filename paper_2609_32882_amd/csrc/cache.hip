// Writing tokens into the paged 8-bit key/value cache and reading them back.
//
// Bound by memory: a value comes in 2 or 4 bytes and goes out in one (or the
// reverse).  A workgroup takes one page of one KV head, in a write its keys or its
// values.  Its 16 groups of D/8 lanes each take four neighbouring tokens 16 t + 4 g .. + 3 (a dword of codes
// per element of V), with a row's 8 elements in each lane; the page goes through
// LDS in its own order, so both sides of the copy are whole lines although K's
// and V's elements change places.
#include "common.hpp"

namespace vsa2 {

namespace {

__device__ __forceinline__ void load8(float* x, const bf16_t* p) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(float* x, const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(const float* x, bf16_t* p) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]),
                                              pack2_bf16(x[4], x[5]), pack2_bf16(x[6], x[7]));
}
__device__ __forceinline__ void store8(const float* x, float* p) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

__device__ __forceinline__ bool finite_f32(float x) {
    return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u;
}

// Largest over the LPR lanes of a row, in every one of them.
template <int LPR>
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, dpp_f32<0xB1>(x));
    x = fmaxf(x, dpp_f32<0x4E>(x));
    x = fmaxf(x, dpp_f32<0x141>(x));
    if constexpr (LPR == 16) x = fmaxf(x, dpp_f32<0x140>(x));
    return x;
}

// Codes of a row's 8 elements in this lane (two dwords) and the row's power.
// The power is a shift of the exponent, so scaling is exact and the one
// rounding is the conversion's.  448 = 1.75 * 2^8: the smallest e with
// top <= 448 * 2^e is top's exponent less 8, and one more above 1.75.
template <int LPR>
__device__ __forceinline__ int quantise8(const float* x, uint32_t* code) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_f32(x[i]) ? fabsf(x[i]) : 0.f);
    const uint32_t bits = __float_as_uint(row_max<LPR>(top));
    int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < -100 ? -100 : e;          // a finite top needs no more than 120
    const float scale = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = finite_f32(x[i]) ? x[i] * scale : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
        code[i] = static_cast<uint32_t>(w);
    }
    return e;
}

struct copy_args {
    cache_view c;
    row_view k, v;
    const int32_t* start;
    const int32_t* count;
    int n, chunks;       // tokens of the call; pages one sequence's tokens can touch
};

// The page a workgroup works on and its tokens' places.
struct page_place {
    int b, h;
    int64_t pos0;        // list position of the page's first token
    int64_t first;       // list position of the call's token 0
    int live_lo, live_hi;   // in-page tokens [lo, hi) that are the call's
    int all_lo, all_hi;     // the same without the sequence's count
    char* page;          // null when the list has no such page
};

template <int D>
__device__ __forceinline__ page_place find_page(const copy_args& a) {
    page_place p;
    const uint32_t item = blockIdx.x, bh = item / a.chunks, chunk = item - bh * a.chunks;
    p.b = static_cast<int>(bh / a.c.heads);
    p.h = static_cast<int>(bh - static_cast<uint32_t>(p.b) * a.c.heads);
    p.first = a.start[p.b];
    int64_t cnt = a.n;
    if (a.count) {
        const int64_t v = a.count[p.b];
        cnt = v < 0 ? 0 : (v < cnt ? v : cnt);
    }
    const int64_t page = (p.first >> 6) + chunk;
    p.pos0 = page << 6;
    auto in_page = [&](int64_t x) { return static_cast<int>(x < 0 ? 0 : (x > 64 ? 64 : x)); };
    p.live_lo = p.all_lo = in_page(p.first - p.pos0);
    p.live_hi = in_page(p.first + cnt - p.pos0);
    p.all_hi = in_page(p.first + a.n - p.pos0);
    p.page = nullptr;
    if (page >= 0 && page < a.c.max_pages && p.live_hi > p.live_lo) {
        const int64_t list = static_cast<int64_t>(p.b) * a.c.table_heads + (a.c.table_heads > 1 ? p.h : 0);
        const int id = a.c.table[list * a.c.max_pages + page];
        if (id >= 0 && id < a.c.pages)
            p.page = a.c.pool + (static_cast<int64_t>(id) * a.c.heads + p.h) * cache_page_bytes(D);
    }
    return p;
}

// blockIdx.y: 0 writes keys, 1 values (half a page each: with whole pages every
// workgroup of a few thousand tokens is resident at once, and all reads come
// before all writes: 7,000 tokens of 12 heads 19.3 us, halves 17.4, 3.7 TB/s).
template <typename T, int D>
__global__ __launch_bounds__(2 * D) void cache_write_kernel(copy_args a) {
    constexpr int LPR = D / 8, CODES = 64 * D, NT = 2 * D;
    __shared__ uint4 image[(CODES + 64) / 16];       // codes, then powers
    const page_place p = find_page<D>(a);
    if (!p.page) return;
    const bool values = blockIdx.y != 0;
    char* lds = reinterpret_cast<char*>(image);
    char* codes = p.page + (values ? CODES : 0);
    char* powers = p.page + 2 * CODES + (values ? 64 : 0);
    const int tid = threadIdx.x, c = tid % LPR, quad = tid / LPR, t = quad >> 2, g = quad & 3;
    const int j0 = 16 * t + 4 * g;
    const row_view& v = values ? a.v : a.k;
    const T* rows = static_cast<const T*>(v.ptr) + p.b * v.batch + p.h * v.head + 8 * c;
    float x[4][8] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (j0 + i >= p.live_lo && j0 + i < p.live_hi) load8(x[i], rows + (p.pos0 + j0 + i - p.first) * v.token);
    uint32_t code[4][2];
    int e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = quantise8<LPR>(x[i], code[i]);
    if (values) {
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w |= ((code[i][d >> 2] >> (8 * (d & 3))) & 0xffu) << (8 * i);
            const int el = 8 * c + d;
            *reinterpret_cast<uint32_t*>(lds + ((el / 16) * 64 + g * 16 + el % 16) * 16 + t * 4) = w;
        }
        if (c == 0)
            *reinterpret_cast<uint32_t*>(lds + CODES + g * 16 + t * 4) =
                static_cast<uint32_t>(e[0] + 127) | static_cast<uint32_t>(e[1] + 127) << 8 |
                static_cast<uint32_t>(e[2] + 127) << 16 | static_cast<uint32_t>(e[3] + 127) << 24;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = ((t * (D / 64) + c / 8) * 64 + (c % 8) / 2 * 16 + 4 * g + i) * 16 + (c & 1) * 8;
            *reinterpret_cast<uint2*>(lds + at) = make_uint2(code[i][0], code[i][1]);
            if (c == 0) lds[CODES + (4 * g + i) * 4 + t] = static_cast<char>(e[i] + 127);
        }
    }
    __syncthreads();
    uint4* out = reinterpret_cast<uint4*>(codes);
    if (p.live_hi - p.live_lo == 64) {
        for (int u = tid; u < CODES / 16; u += NT) out[u] = image[u];
        if (tid < 4) reinterpret_cast<uint4*>(powers)[tid] = image[CODES / 16 + tid];
        return;
    }
    // part of a page: the bytes of the call's tokens alone, the others are other calls'
    const uint64_t live = (p.live_hi == 64 ? ~0ull : (1ull << p.live_hi) - 1) & ~((1ull << p.live_lo) - 1);
    const auto four = [&](char* to, int at, uint32_t bytes) {       // the marked bytes of a dword
        if (bytes == 15u) {
            *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(lds + at);
        } else if (bytes) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((bytes >> i) & 1) to[i] = lds[at + i];
        }
    };
    if (values) {                                       // dword: tokens 16 tt + 4 gg + i
        for (int w = tid; w < 16 * D + 16; w += NT) {
            const int tt = w & 3, gg = w < 16 * D ? (w >> 6) & 3 : ((w - 16 * D) >> 2) & 3;
            four(w < 16 * D ? codes + 4 * w : powers + 4 * (w - 16 * D), 4 * w,
                 static_cast<uint32_t>(live >> (16 * tt + 4 * gg)) & 15u);
        }
    } else {
        for (int u = tid; u < 4 * D; u += NT) {         // a 16-byte piece is one token's
            const int r = u & 15, tt = u / D;           // D pieces per 16 tokens
            if ((live >> (16 * tt + r)) & 1) out[u] = image[u];
        }
        if (tid < 16) {                                 // powers: tokens 16 i + r
            const uint64_t m = live >> tid;
            four(powers + 4 * tid, CODES + 4 * tid,
                 static_cast<uint32_t>((m & 1) | (m >> 15 & 2) | (m >> 30 & 4) | (m >> 45 & 8)));
        }
    }
}

__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two sequences of 76,800 tokens, 8 heads of 128, into bf16: 195 us, 4.9 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(2 * D) void cache_read_kernel(copy_args a) {
    constexpr int LPR = D / 8, BYTES = static_cast<int>(cache_page_bytes(D)), NT = 2 * D;
    __shared__ uint4 image[BYTES / 16];
    const page_place p = find_page<D>(a);
    const int tid = threadIdx.x, c = tid % LPR, quad = tid / LPR, t = quad >> 2, g = quad & 3;
    if (p.page) {
        const uint4* in = reinterpret_cast<const uint4*>(p.page);
        for (int u = tid; u < BYTES / 16; u += NT) image[u] = in[u];
    }
    __syncthreads();
    const char* lds = reinterpret_cast<const char*>(image);
    uint32_t vcode[8], ve = 0;
    if (p.page) {
        ve = *reinterpret_cast<const uint32_t*>(lds + 128 * D + 64 + g * 16 + t * 4);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const int e = 8 * c + d;
            vcode[d] = *reinterpret_cast<const uint32_t*>(lds + 64 * D + ((e / 16) * 64 + g * 16 + e % 16) * 16 + t * 4);
        }
    }
    T* kp = static_cast<T*>(a.k.ptr) + p.b * a.k.batch + p.h * a.k.head + 8 * c;
    T* vp = static_cast<T*>(a.v.ptr) + p.b * a.v.batch + p.h * a.v.head + 8 * c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 16 * t + 4 * g + i;
        if (j < p.all_lo || j >= p.all_hi) continue;
        const int64_t tok = p.pos0 + j - p.first;
        float k[8] = {}, v[8] = {};
        if (p.page && j < p.live_hi) {
            const int at = ((t * (D / 64) + c / 8) * 64 + (c % 8) / 2 * 16 + 4 * g + i) * 16 + (c & 1) * 8;
            const uint2 kc = *reinterpret_cast<const uint2*>(lds + at);
            const float sk = power_of(static_cast<uint8_t>(lds[128 * D + (4 * g + i) * 4 + t]));
            const float sv = power_of((ve >> (8 * i)) & 0xffu);
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                const uint32_t kw = (d < 4 ? kc.x : kc.y) >> (8 * (d & 3));
                k[d] = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(kw), 0) * sk;
                v[d] = __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(vcode[d] >> (8 * i)), 0) * sv;
            }
        }
        store8(k, kp + tok * a.k.token);
        store8(v, vp + tok * a.v.token);
    }
}

}  // namespace

hipError_t launch_cache_copy(bool write, int dtype, int D, const cache_view& c, int n, const row_view& k,
                             const row_view& v, const int32_t* start, const int32_t* count, hipStream_t s) {
    copy_args a{c, k, v, start, count, n, static_cast<int>((static_cast<int64_t>(n) + 62) / 64 + 1)};
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(c.batch) * c.heads * a.chunks), write ? 2 : 1), block(2 * D);
#define VSA2_CACHE_GO(T, DD)                                                                     \
    do {                                                                                         \
        if (write) hipLaunchKernelGGL((cache_write_kernel<T, DD>), grid, block, 0, s, a);        \
        else hipLaunchKernelGGL((cache_read_kernel<T, DD>), grid, block, 0, s, a);               \
    } while (0)
    if (dtype == 0 && D == 64) VSA2_CACHE_GO(float, 64);
    else if (dtype == 0) VSA2_CACHE_GO(float, 128);
    else if (D == 64) VSA2_CACHE_GO(bf16_t, 64);
    else VSA2_CACHE_GO(bf16_t, 128);
#undef VSA2_CACHE_GO
    return hipGetLastError();
}

}  // namespace vsa2
