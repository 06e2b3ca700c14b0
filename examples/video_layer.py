"""One attention layer of a video model around the library, in training and in
streaming generation, with random weights and inputs.

Training: projection -> per-head norm, (time, height, width) rotation and cube-
major layout in one call -> pool -> route -> block-sparse attention -> its
gradients -> the projection's and the gains' gradients.

Streaming: frames arrive in chunks.  A chunk's tokens stay in raster order
(1 x 1 x 1 cubes), are rotated by their place in the clip, and go into a paged
8-bit cache; the chunk then attends everything the cache holds.

    python examples/video_layer.py
"""
import dataclasses
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2609_32882_amd as vsa2


@dataclasses.dataclass
class Layer:
    heads_q: int = 4
    heads_kv: int = 2
    head_dim: int = 128
    axes: tuple = (44, 42, 42)      # elements of a head turned by time, height, width
    eps: float = 1e-6
    top_k: int = 4
    dtype: torch.dtype = torch.bfloat16
    seed: int = 0

    def __post_init__(self):
        g = torch.Generator(device="cuda").manual_seed(self.seed)
        width, heads = self.heads_q * self.head_dim, self.heads_q + 2 * self.heads_kv
        self.w_qkv = (torch.randn(width, heads * self.head_dim, generator=g, device="cuda") / width ** 0.5).to(self.dtype)
        self.q_gain = 1 + 0.1 * torch.randn(self.head_dim, generator=g, device="cuda")
        self.k_gain = 1 + 0.1 * torch.randn(self.head_dim, generator=g, device="cuda")

    def problem(self, batch, grid, cube):
        return vsa2.make_problem(batch, self.heads_q, self.heads_kv, self.head_dim, *grid, cube, cube, cube,
                                 max(cube // 2, 1), max(cube // 2, 1), max(cube // 2, 1),
                                 vsa2.VSA2_BF16 if self.dtype == torch.bfloat16 else vsa2.VSA2_F32)

    def rope(self, grid, origin=None):
        tables = [vsa2.rope_table(n, a) if a else None for n, a in zip(grid, self.axes)]
        return vsa2.Rope(self.axes, tables, origin)

    def split(self, qkv):
        """q, k, v of the projected rows [batch, tokens, heads * D], [batch, heads, tokens, D] each."""
        x = qkv.view(*qkv.shape[:2], -1, self.head_dim)
        return [y.transpose(1, 2) for y in x.split([self.heads_q, self.heads_kv, self.heads_kv], 2)]

    def training_step(self, x, dout, grid):
        """x [batch, tokens, width] in raster order, dout the gradient of the attention's
        output [batch, heads_q, L, D]: (output, gradients of w_qkv, q_gain, k_gain)."""
        p, rope = self.problem(x.shape[0], grid, 4), self.rope(grid)
        qkv = x @ self.w_qkv
        raw = self.split(qkv)
        norm = dict(q_gain=self.q_gain, k_gain=self.k_gain, rope=rope, eps=self.eps)
        q, k, v = vsa2.qk_norm_rope(p, *raw, **norm)
        pooled = [vsa2.pool(p, t, (p.Rt, p.Rh, p.Rw)) for t in (q, k)]
        r = vsa2.route(p, vsa2.vsa2_select(vsa2.VSA2_SEL_TOPK, self.top_k, 0.0, 0), *pooled)
        o, lse, o_lo = vsa2.attn_fwd(p, q, k, v, r["row_ptr"], r["col_idx"], training=True)
        dq, dk, dv = vsa2.attn_bwd(p, q, k, v, o, lse, dout, r["row_ptr"], r["col_idx"], r["kv_ptr"], r["kv_idx"],
                                   o_lo=o_lo)
        d_qkv = torch.empty_like(qkv)
        *_, dq_gain, dk_gain = vsa2.qk_norm_rope_bwd(p, dq, dk, dv, q=raw[0], k=raw[1], out=self.split(d_qkv), **norm)
        dw = x.flatten(0, 1).t() @ d_qkv.flatten(0, 1)
        return o, dw, dq_gain, dk_gain

    def stream(self, chunks, grid):
        """chunks: [batch, frames * h * w, width] each, frames of grid = (frames of the whole
        clip, h, w) in order.  Yields each chunk's attention output [batch, tokens, heads_q * D]."""
        batch, (frames, h, w) = chunks[0].shape[0], grid
        pages = -(-frames * h * w // 64)
        table = torch.arange(batch * pages, dtype=torch.int32, device="cuda").view(batch, pages)
        cache = vsa2.KVCache.empty(table, batch * pages, self.heads_kv, self.head_dim)
        start = torch.zeros(batch, dtype=torch.int32, device="cuda")
        origin = torch.zeros(batch, 3, dtype=torch.int32, device="cuda")
        rope = self.rope(grid, origin)
        for x in chunks:
            n = x.shape[1]
            p = self.problem(batch, (n // (h * w), h, w), 1)
            q, k, v = self.split(x @ self.w_qkv)
            q, k, _ = vsa2.qk_norm_rope(p, q, k, q_gain=self.q_gain, k_gain=self.k_gain, rope=rope, eps=self.eps)
            vsa2.cache_write(cache, k, v, start)
            start += n
            origin[:, 0] += n // (h * w)
            o = torch.empty(batch, n, self.heads_q, self.head_dim, dtype=x.dtype, device="cuda")
            vsa2.attn_cache(cache, q, start, o=o.transpose(1, 2))
            yield o.flatten(2)


def main():
    layer, grid = Layer(), (8, 16, 16)
    g = torch.Generator(device="cuda").manual_seed(1)
    width = layer.heads_q * layer.head_dim
    x = torch.randn(1, 8 * 16 * 16, width, generator=g, device="cuda").to(layer.dtype)
    dout = torch.randn(1, layer.heads_q, 8 * 16 * 16, layer.head_dim, generator=g, device="cuda").to(layer.dtype)
    o, dw, dq_gain, dk_gain = layer.training_step(x, dout, grid)
    print("training step: output %s, |dW| %.3g, |dq_gain| %.3g, |dk_gain| %.3g" %
          (tuple(o.shape), dw.float().norm(), dq_gain.norm(), dk_gain.norm()))
    for i, y in enumerate(layer.stream(x.split([1 * 256, 3 * 256, 4 * 256], 1), grid)):
        print("chunk %d: %d tokens, |output| %.3g" % (i, y.shape[1], y.float().norm()))


if __name__ == "__main__":
    main()
