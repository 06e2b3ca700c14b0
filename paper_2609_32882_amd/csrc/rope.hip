// Per-head RMS norm of queries and keys, rotation by the token's position and
// the cube-major layout in one pass, and its gradients.
//
// Bound by memory: an element is read once and written once and takes about 7
// operations (14 in the gradients).  A row of D elements lies in D/8 lanes of
// 8 elements, so a wave holds RPW = 512/D rows of consecutive cube-major tokens
// (4 at D = 128: one run of a 4 x 4 x 4 cube, whose output rows are 1 KB in a
// piece).  What depends on the token alone (its place, its sequence, its 4
// (cos, sin) pairs) is worked out once per lane and kept while the wave walks
// over the heads; neighbouring waves take neighbouring heads, whose input rows
// lie side by side in a projection.  A 20x48x80 grid with 40 + 40 + 40 heads of
// 128 in bf16 takes 930 us (5.0 TB/s, a large copy's rate); its gradients with
// 12 + 12 + 12 heads 375 us (5.0 TB/s).
#include "common.hpp"

namespace vsa2 {

namespace {

// 8 elements of one row as they came from memory.
template <typename T> struct raw8;
template <> struct raw8<bf16_t> { uint2 a, b; };
template <> struct raw8<float> { float4 a, b; };

// Elements a0 .. a0+3 and a1 .. a1+3 of a row (one 32-byte or 16-byte run when
// a1 = a0 + 4).
template <bool RUN>
__device__ __forceinline__ void load_raw(raw8<bf16_t>& r, const bf16_t* row, int a0, int a1) {
    if constexpr (RUN) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + a0);
        r.a = make_uint2(w.x, w.y);
        r.b = make_uint2(w.z, w.w);
    } else {
        r.a = *reinterpret_cast<const uint2*>(row + a0);
        r.b = *reinterpret_cast<const uint2*>(row + a1);
    }
}
template <bool RUN>
__device__ __forceinline__ void load_raw(raw8<float>& r, const float* row, int a0, int a1) {
    r.a = *reinterpret_cast<const float4*>(row + a0);
    r.b = *reinterpret_cast<const float4*>(row + a1);
}
template <bool RUN>
__device__ __forceinline__ void store_raw(const raw8<bf16_t>& r, bf16_t* row, int a0, int a1) {
    if constexpr (RUN) {
        *reinterpret_cast<uint4*>(row + a0) = make_uint4(r.a.x, r.a.y, r.b.x, r.b.y);
    } else {
        *reinterpret_cast<uint2*>(row + a0) = r.a;
        *reinterpret_cast<uint2*>(row + a1) = r.b;
    }
}
template <bool RUN>
__device__ __forceinline__ void store_raw(const raw8<float>& r, float* row, int a0, int a1) {
    *reinterpret_cast<float4*>(row + a0) = r.a;
    *reinterpret_cast<float4*>(row + a1) = r.b;
}

// The 4 pairs (x0, x1) a lane holds: neighbouring elements of its run, or
// element i of each half.
template <bool HALVES>
__device__ __forceinline__ void to_pairs(const raw8<bf16_t>& r, float* x0, float* x1) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.b.x, r.b.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
        if constexpr (HALVES) {
            float* x = i < 2 ? x0 : x1;
            x[2 * (i & 1)] = lo;
            x[2 * (i & 1) + 1] = hi;
        } else {
            x0[i] = lo;
            x1[i] = hi;
        }
    }
}
template <bool HALVES>
__device__ __forceinline__ void to_pairs(const raw8<float>& r, float* x0, float* x1) {
    const float v[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x0[i] = HALVES ? v[i] : v[2 * i];
        x1[i] = HALVES ? v[4 + i] : v[2 * i + 1];
    }
}
template <bool HALVES>
__device__ __forceinline__ void from_pairs(raw8<bf16_t>& r, const float* x0, const float* x1) {
    if constexpr (HALVES) {
        r.a = make_uint2(pack2_bf16(x0[0], x0[1]), pack2_bf16(x0[2], x0[3]));
        r.b = make_uint2(pack2_bf16(x1[0], x1[1]), pack2_bf16(x1[2], x1[3]));
    } else {
        r.a = make_uint2(pack2_bf16(x0[0], x1[0]), pack2_bf16(x0[1], x1[1]));
        r.b = make_uint2(pack2_bf16(x0[2], x1[2]), pack2_bf16(x0[3], x1[3]));
    }
}
template <bool HALVES>
__device__ __forceinline__ void from_pairs(raw8<float>& r, const float* x0, const float* x1) {
    if constexpr (HALVES) {
        r.a = make_float4(x0[0], x0[1], x0[2], x0[3]);
        r.b = make_float4(x1[0], x1[1], x1[2], x1[3]);
    } else {
        r.a = make_float4(x0[0], x1[0], x0[1], x1[1]);
        r.b = make_float4(x0[2], x1[2], x0[3], x1[3]);
    }
}

// Sum over the LPR (8 or 16) lanes of a row, in every one of them.
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
    x += dpp_f32<0xB1>(x);      // quad_perm 1 0 3 2
    x += dpp_f32<0x4E>(x);      // quad_perm 2 3 0 1
    x += dpp_f32<0x141>(x);     // row_half_mirror: the other quad of 8
    if constexpr (LPR == 16) x += dpp_f32<0x140>(x);   // row_mirror: the other 8 of 16
    return x;
}

// What a lane knows of its token, whatever the head.
struct lane_token {
    int64_t b;       // sequence
    int64_t l;       // place in the cube-major order
    int64_t at;      // raster token, -1 for padding
    bool valid;      // the row exists
    float c[4], s[4];
};

template <bool HALVES>
__device__ __forceinline__ lane_token find_token(const rope_args& a, int64_t flat, int c) {
    lane_token t;
    const uint32_t Lj = static_cast<uint32_t>(a.Lj);
    t.valid = flat < a.tokens;
    const uint32_t f = t.valid ? static_cast<uint32_t>(flat) : 0u;
    const uint32_t b = f / Lj, l = f - b * Lj;
    t.b = b;
    t.l = l;
    const cube_grid& g = a.grid;
    const uint32_t B = static_cast<uint32_t>(g.Bt) * g.Bh * g.Bw;
    const uint32_t n = l / B, beta = l - n * B;
    int pos[3] = {0, 0, 0};
    bool turned = false;
    if (n < static_cast<uint32_t>(g.Nv)) {
        const uint32_t nr = n / g.Nw, nw = n - nr * g.Nw, nt = nr / g.Nh, nh = nr - nt * g.Nh;
        const uint32_t br = beta / g.Bw, bw = beta - br * g.Bw, bt = br / g.Bh, bh = br - bt * g.Bh;
        const int pt = static_cast<int>(nt * g.Bt + bt), ph = static_cast<int>(nh * g.Bh + bh),
                  pw = static_cast<int>(nw * g.Bw + bw);
        const bool real = pt < g.T && ph < g.H && pw < g.W;
        t.at = real ? (static_cast<int64_t>(pt) * g.H + ph) * g.W + pw : -1;
        turned = real;
        pos[0] = pt;
        pos[1] = ph;
        pos[2] = pw;
    } else {
        const int64_t i = static_cast<int64_t>(l) - static_cast<int64_t>(g.Nv) * B;
        t.at = i < g.text_len ? static_cast<int64_t>(g.T) * g.H * g.W + i : -1;
    }
    if (!t.valid) t.at = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t.c[i] = 1.f;
        t.s[i] = 0.f;
    }
    if (turned && t.valid) {
        int first = 0;                          // the axis' first pair
#pragma unroll
        for (int x = 0; x < 3; ++x) {
            const int np = a.axis_pairs[x];
            if (np > 0) {
                // a sequence's origin may be anything: clamped into the table
                int64_t row = static_cast<int64_t>(pos[x]) + (a.origin ? a.origin[t.b * 3 + x] : 0);
                row = row < 0 ? 0 : (row >= a.table_rows[x] ? a.table_rows[x] - 1 : row);
                const float2* tab = reinterpret_cast<const float2*>(a.table[x]) + row * np - first;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int pair = 4 * c + i;
                    if (pair >= first && pair < first + np) {
                        const float2 cs = tab[pair];
                        t.c[i] = cs.x;
                        t.s[i] = cs.y;
                    }
                }
                first += np;
            }
        }
    }
    return t;
}

// First elements of a lane's two runs of 4.  HALVES: element i of both halves
// of the turned part, then plain runs of 8 past it.
template <bool HALVES>
__device__ __forceinline__ void lane_runs(int pairs, int c, int& a0, int& a1) {
    if (HALVES && 4 * c < pairs) {
        a0 = 4 * c;
        a1 = pairs + 4 * c;
    } else {
        a0 = 8 * c;
        a1 = 8 * c + 4;
    }
}

__device__ __forceinline__ void load_gain(float* g0, float* g1, const float* gain, int a0, int a1, bool halves) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g0[i] = !gain ? 1.f : gain[halves ? a0 + i : a0 + 2 * i];
        g1[i] = !gain ? 1.f : gain[halves ? a1 + i : a0 + 2 * i + 1];
    }
}

// Which part (0 q, 1 k, 2 v) head hh of all parts' heads is in, and its index there.
__device__ __forceinline__ int part_of(const rope_args& a, int hh, int& h) {
    int x = 0;
    h = hh;
    if (h >= a.part[0].heads) { h -= a.part[0].heads; x = 1; }
    if (x == 1 && h >= a.part[1].heads) { h -= a.part[1].heads; x = 2; }
    return x;
}

template <typename T>
__device__ __forceinline__ const T* row_at(const row_view& r, const lane_token& t, int h) {
    return static_cast<const T*>(r.ptr) + t.b * r.batch + h * r.head + t.at * r.token;
}

constexpr int ROPE_WAVES = 4;
constexpr int ROPE_AHEAD = 4;     // heads whose rows are requested together

template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(64 * ROPE_WAVES) void norm_rope_kernel(rope_args a) {
    constexpr int LPR = D / 8, RPW = 64 / LPR;
    const int lane = lane_id(), c = lane % LPR, rr = lane / LPR;
    const lane_token t = find_token<HALVES>(a, static_cast<int64_t>(blockIdx.x) * RPW + rr, c);
    int a0, a1;
    lane_runs<HALVES>(a.pairs, c, a0, a1);
    float gain[2][2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) load_gain(gain[x][0], gain[x][1], a.part[x].gain, a0, a1, HALVES);
    const int stride = ROPE_WAVES * gridDim.y, slot = blockIdx.y * ROPE_WAVES + wave_id();
    const int heads = a.part[0].heads + a.part[1].heads + a.part[2].heads;
    for (int h0 = slot; h0 < heads; h0 += stride * ROPE_AHEAD) {
        raw8<T> raw[ROPE_AHEAD];
#pragma unroll
        for (int u = 0; u < ROPE_AHEAD; ++u) {
            int h;
            const int hh = h0 + u * stride;
            raw[u] = raw8<T>{};
            if (hh < heads && t.at >= 0) {
                const row_view& in = a.part[part_of(a, hh, h)].x;
                load_raw<!HALVES>(raw[u], row_at<T>(in, t, h), a0, a1);
            }
        }
#pragma unroll
        for (int u = 0; u < ROPE_AHEAD; ++u) {
            int h;
            const int hh = h0 + u * stride;
            if (hh >= heads) break;
            const int x = part_of(a, hh, h);
            if (x < 2) {
                float x0[4], x1[4];
                to_pairs<HALVES>(raw[u], x0, x1);
                if (a.eps > 0.f) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) ss = fmaf(x0[i], x0[i], fmaf(x1[i], x1[i], ss));
                    const float r = rsqrtf(row_sum<LPR>(ss) * (1.f / D) + a.eps);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x0[i] = x0[i] * r * (x == 0 ? gain[0][0][i] : gain[1][0][i]);
                        x1[i] = x1[i] * r * (x == 0 ? gain[0][1][i] : gain[1][1][i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y0 = x0[i] * t.c[i] - x1[i] * t.s[i];
                    x1[i] = x0[i] * t.s[i] + x1[i] * t.c[i];
                    x0[i] = y0;
                }
                from_pairs<HALVES>(raw[u], x0, x1);
            }
            if (t.valid) {
                const rope_part& p = a.part[x];
                T* out = static_cast<T*>(p.y) + ((t.b * p.heads + h) * a.Lj + t.l) * D;
                store_raw<!HALVES>(raw[u], out, a0, a1);
            }
        }
    }
}

// The norm's gradient in place: g with respect to the gained row -> to x; adds
// the row's part of the gain's gradient to dg.
template <int D>
__device__ __forceinline__ void norm_back(float (&g0)[4], float (&g1)[4], float (&x0)[4], float (&x1)[4], float eps,
                                          const float (&w)[2][4], float (&dg)[2][4]) {
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) ss = fmaf(x0[i], x0[i], fmaf(x1[i], x1[i], ss));
    const float r = rsqrtf(row_sum<D / 8>(ss) * (1.f / D) + eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x0[i] *= r;
        x1[i] *= r;
        const float e0 = g0[i] * x0[i], e1 = g1[i] * x1[i];
        dg[0][i] += e0;
        dg[1][i] += e1;
        dot = fmaf(e0, w[0][i], fmaf(e1, w[1][i], dot));
        g0[i] *= w[0][i];
        g1[i] *= w[1][i];
    }
    const float mean = row_sum<D / 8>(dot) * (1.f / D);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g0[i] = r * (g0[i] - x0[i] * mean);
        g1[i] = r * (g1[i] - x1[i] * mean);
    }
}

// Gradients.  The gains' gradients are sums over every token and head: each
// lane adds up its 8 elements over the tokens and heads its wave walks over,
// the workgroup joins its waves and rows in LDS and writes one partial row
// [2][D], and norm_rope_gain_kernel adds the workgroups' rows in their order.
// Grid and order depend on the sizes alone, so the sums are reproducible.
template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(64 * ROPE_WAVES) void norm_rope_bwd_kernel(rope_args a) {
    constexpr int LPR = D / 8, RPW = 64 / LPR;
    const int lane = lane_id(), c = lane % LPR, rr = lane / LPR;
    int a0, a1;
    lane_runs<HALVES>(a.pairs, c, a0, a1);
    float gain[2][2][4], dg[2][2][4] = {};
#pragma unroll
    for (int x = 0; x < 2; ++x) load_gain(gain[x][0], gain[x][1], a.part[x].gain, a0, a1, HALVES);
    const int stride = ROPE_WAVES * gridDim.y, slot = blockIdx.y * ROPE_WAVES + wave_id();
    const int heads = a.part[0].heads + a.part[1].heads + a.part[2].heads;
    const bool norm = a.eps > 0.f;
    const int64_t groups = (a.tokens + RPW - 1) / RPW;
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const lane_token t = find_token<HALVES>(a, group * RPW + rr, c);
        constexpr int AHEAD = 2;       // three or four: fp32 255 -> 305 us (20x48x40, 8 heads), bf16 the same
        for (int h0 = slot; h0 < heads; h0 += stride * AHEAD) {
            raw8<T> rg[AHEAD], rx[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                int h;
                const int hh = h0 + u * stride;
                rg[u] = rx[u] = raw8<T>{};
                if (hh < heads && t.at >= 0) {
                    const int x = part_of(a, hh, h);
                    const rope_part& p = a.part[x];
                    const T* dy = static_cast<const T*>(p.y) + ((t.b * p.heads + h) * a.Lj + t.l) * D;
                    load_raw<!HALVES>(rg[u], dy, a0, a1);
                    if (norm && x < 2) load_raw<!HALVES>(rx[u], row_at<T>(p.x, t, h), a0, a1);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                int h;
                const int hh = h0 + u * stride;
                const int x = part_of(a, hh, h);
                if (hh < heads && x < 2) {
                    float g0[4], g1[4];
                    to_pairs<HALVES>(rg[u], g0, g1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float b0 = g0[i] * t.c[i] + g1[i] * t.s[i];
                        g1[i] = g1[i] * t.c[i] - g0[i] * t.s[i];
                        g0[i] = b0;
                    }
                    if (norm) {
                        float x0[4], x1[4];
                        to_pairs<HALVES>(rx[u], x0, x1);
                        if (x == 0) norm_back<D>(g0, g1, x0, x1, a.eps, gain[0], dg[0]);
                        else norm_back<D>(g0, g1, x0, x1, a.eps, gain[1], dg[1]);
                    }
                    from_pairs<HALVES>(rg[u], g0, g1);
                }
                if (hh < heads && t.at >= 0) {
                    const row_view& out = a.part[x].dx;
                    store_raw<!HALVES>(rg[u], const_cast<T*>(row_at<T>(out, t, h)), a0, a1);
                }
            }
        }
    }
    if (!a.partial) return;
    __shared__ float part[ROPE_WAVES * RPW][2][D];
    const int at = wave_id() * RPW + rr;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            part[at][x][HALVES ? a0 + i : a0 + 2 * i] = dg[x][0][i];
            part[at][x][HALVES ? a1 + i : a0 + 2 * i + 1] = dg[x][1][i];
        }
    __syncthreads();
    const int64_t wg = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
    for (int i = threadIdx.x; i < 2 * D; i += blockDim.x) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < ROPE_WAVES * RPW; ++w) sum += part[w][i / D][i % D];
        a.partial[wg * 2 * D + i] = sum;
    }
}

// Column sums of the partial rows [n][2 D]: a workgroup takes 16 columns, its
// 64 groups of 16 lanes every 64th row each, four rows in flight.
__global__ __launch_bounds__(1024) void norm_rope_gain_kernel(const float* partial, int64_t n, int D, float* dq_gain,
                                                              float* dk_gain) {
    __shared__ float part[64][16];
    const int lane = threadIdx.x & 15, slice = threadIdx.x >> 4, col = blockIdx.x * 16 + lane;
    float sum[4] = {};
    for (int64_t r = slice; r < n; r += 4 * 64) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (r + 64 * u < n) sum[u] += partial[(r + 64 * u) * 2 * D + col];
    }
    part[slice][lane] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    __syncthreads();
    if (threadIdx.x < 16) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < 64; ++w) total += part[w][lane];
        float* out = col < D ? dq_gain : dk_gain;
        if (out) out[col < D ? col : col - D] = total;
    }
}

// Workgroups along the heads, so that a few tokens still fill the CUs.
int head_split(int64_t groups, int heads) {
    const int64_t want = (1024 + groups - 1) / groups, most = (heads + ROPE_WAVES - 1) / ROPE_WAVES;
    return static_cast<int>(want > most ? most : want);
}

// Workgroups along the tokens in the gradients: each writes one partial row.
constexpr int64_t BWD_GROUPS = 1024;

}  // namespace

size_t norm_rope_workspace_bytes(int D, int64_t tokens, int heads) {
    const int rpw = 512 / D;
    const int64_t groups = (tokens + rpw - 1) / rpw, gx = groups < BWD_GROUPS ? groups : BWD_GROUPS;
    return static_cast<size_t>(gx) * head_split(groups, heads) * 2 * D * sizeof(float);
}

#define VSA2_ROPE_DISPATCH(KERNEL, GRID)                                                                       \
    do {                                                                                                       \
        const dim3 block(64 * ROPE_WAVES);                                                                     \
        if (dtype == 0 && D == 64 && !halves) hipLaunchKernelGGL((KERNEL<float, 64, false>), GRID, block, 0, s, a);        \
        else if (dtype == 0 && D == 64) hipLaunchKernelGGL((KERNEL<float, 64, true>), GRID, block, 0, s, a);               \
        else if (dtype == 0 && !halves) hipLaunchKernelGGL((KERNEL<float, 128, false>), GRID, block, 0, s, a);             \
        else if (dtype == 0) hipLaunchKernelGGL((KERNEL<float, 128, true>), GRID, block, 0, s, a);                         \
        else if (D == 64 && !halves) hipLaunchKernelGGL((KERNEL<bf16_t, 64, false>), GRID, block, 0, s, a);                \
        else if (D == 64) hipLaunchKernelGGL((KERNEL<bf16_t, 64, true>), GRID, block, 0, s, a);                            \
        else if (!halves) hipLaunchKernelGGL((KERNEL<bf16_t, 128, false>), GRID, block, 0, s, a);                          \
        else hipLaunchKernelGGL((KERNEL<bf16_t, 128, true>), GRID, block, 0, s, a);                                        \
    } while (0)

hipError_t launch_norm_rope(int dtype, int D, bool halves, const rope_args& a, hipStream_t s) {
    const int heads = a.part[0].heads + a.part[1].heads + a.part[2].heads;
    if (heads == 0) return hipSuccess;
    const int rpw = 512 / D;
    const int64_t groups = (a.tokens + rpw - 1) / rpw;
    const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>(head_split(groups, heads)));
    VSA2_ROPE_DISPATCH(norm_rope_kernel, grid);
    return hipGetLastError();
}

hipError_t launch_norm_rope_bwd(int dtype, int D, bool halves, const rope_args& a, float* dq_gain, float* dk_gain,
                                hipStream_t s) {
    const int heads = a.part[0].heads + a.part[1].heads + a.part[2].heads;
    if (heads == 0) return hipSuccess;
    const int rpw = 512 / D;
    const int64_t groups = (a.tokens + rpw - 1) / rpw, gx = groups < BWD_GROUPS ? groups : BWD_GROUPS;
    const int gy = head_split(groups, heads);
    const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>(gy));
    VSA2_ROPE_DISPATCH(norm_rope_bwd_kernel, grid);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partial) return e;
    hipLaunchKernelGGL(norm_rope_gain_kernel, dim3(2 * D / 16), dim3(1024), 0, s, a.partial, gx * gy, D, dq_gain,
                       dk_gain);
    return hipGetLastError();
}
#undef VSA2_ROPE_DISPATCH

}  // namespace vsa2
