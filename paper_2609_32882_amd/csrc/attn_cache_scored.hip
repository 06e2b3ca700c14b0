// Attention of new tokens over the paged 8-bit cache with capped scores, a bias by
// distance, a window behind some first positions, and a range of positions for every
// token.
//
// The plain attention's kernels with two changes.  A page's scores become
//   log2 e (cap tanh(x / cap) - slope |at - j|)
// between the two products, in the registers that hold them.  And rows see two ranges of
// positions, [0, sinks) and [lo, hi): a workgroup visits the pages from the list's
// start to the rows' last sink, then those of their ranges together; pages that every
// row sees whole take the step without masks.  Inside the others a lane makes a bit for
// each of its tokens; what no row of a tile sees may never have been written, so its
// powers do not count for the scale of P and its codes are zeros.
//
// One token each of 16 sequences over up to 38,400, 40/8 heads of 128, capped: 156 us, 5.3
// TB/s, bound by memory as the plain attention.  1,792 tokens over the first 1,792 and the last
// 8,960 positions, 12 heads, cap and bias: 209 to 216 us with the card's clock, 0.6 PFLOP/s, bound by
// vector instructions beside the MFMAs (61% and 25% of a SIMD's cycles); a loop that goes back and forth between
// pages with and without masks, compiled for each, spilled 222 registers more and took 271.
#include <algorithm>

#include "cache_tile.hpp"

namespace vsa2 {

namespace {

template <typename T, int D, int WAVES, int XT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, D == 128 ? 2 : 4))) void scored_tiles_kernel(
    attn_args a, scored sc) {
    __shared__ tile_lds<D, WAVES, XT> lds;
    tile_body<T, D, WAVES, XT, WHOLE>(a, sc, blockIdx.x, gridDim.x, lds);
}
template <typename T, int D>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 4 ? 1 : 2) void scored_rows_kernel(attn_args a, scored sc) {
    __shared__ rows_lds<D> lds;
    rows_body<T, D, WHOLE>(a, sc, blockIdx.x, gridDim.x, lds);
}

struct scored_kernels {
    scored sc;
    template <typename T, int D, int WAVES, int XT>
    void tiles(dim3 grid, dim3 block, hipStream_t s, const attn_args& a) const {
        hipLaunchKernelGGL((scored_tiles_kernel<T, D, WAVES, XT>), grid, block, 0, s, a, sc);
    }
    template <typename T, int D>
    void rows(dim3 grid, dim3 block, hipStream_t s, const attn_args& a) const {
        hipLaunchKernelGGL((scored_rows_kernel<T, D>), grid, block, 0, s, a, sc);
    }
};

// The pages that a call's rows may see at most, for the plan: with a window, that of its
// tokens together and the first positions.
cache_view window_view(const cache_view& c, int n, int window, int sink) {
    cache_view v = c;
    if (window) {
        const int64_t most = static_cast<int64_t>(window) + n + 2 * CACHE_TOKENS + sink + CACHE_TOKENS;
        v.max_pages = static_cast<int>(std::min<int64_t>(c.max_pages, most / CACHE_TOKENS));
    }
    return v;
}

}  // namespace

size_t attn_cache_scored_workspace_bytes(const cache_view& c, int D, int heads_q, int n, int window, int sink) {
    return attn_cache_workspace_bytes(window_view(c, n, window, sink), D, heads_q, n);
}

hipError_t launch_attn_cache_scored(int dtype, int D, const cache_view& c, int heads_q, int n, const row_view& q,
                                    const int32_t* length, const int32_t* count, bool causal, const score_options& options,
                                    const row_view& o, float* lse, void* ws, hipStream_t s) {
    const attn_plan p = plan_attn(dtype, D, window_view(c, n, options.window, options.sink), heads_q, n);
    const attn_args a = plan_args(p, c, heads_q, n, q, length, count, causal, o, lse, ws);
    const scored_kernels go{scored{options}};
    if (dtype == 0 && D == 64) launch_attn<float, 64>(a, p, s, go);
    else if (dtype == 0) launch_attn<float, 128>(a, p, s, go);
    else if (D == 64) launch_attn<bf16_t, 64>(a, p, s, go);
    else launch_attn<bf16_t, 128>(a, p, s, go);
    return hipGetLastError();
}

}  // namespace vsa2
