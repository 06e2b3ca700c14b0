"""examples/video_layer.py: the operators together, against a plain layer."""
import math
import os
import sys

import pytest
import torch

import around_reference as ref

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain(layer, x, w, gains, grid):
    """q, k, v [heads, tokens, D] in 64 bits: projection, norm, rotation in raster order."""
    import paper_2609_32882_amd as vsa2
    p = layer.problem(1, grid, 1)
    where = ref.place_of(p)[1]
    tables = [vsa2.rope_table(n, a, device="cpu") for n, a in zip(grid, layer.axes)]
    cs = ref.turn_of(p, layer.axes, tables, None, where)
    y = (x @ w).view(1, -1, layer.heads_q + 2 * layer.heads_kv, layer.head_dim).transpose(1, 2)
    q, k, v = y.split([layer.heads_q, layer.heads_kv, layer.heads_kv], 1)
    q, k = (rotate(ref.norm_of(t, g, layer.eps), cs) for t, g in zip((q, k), gains))
    return q[0], k[0], v[0]


def rotate(u, cs):
    """Adjacent pairs turned, without writing in place (autograd follows)."""
    c, s = (t[:, None] for t in cs)
    a, b = u[..., ::2], u[..., 1::2]
    return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)


def attend(layer, q, k, v):
    group = layer.heads_q // layer.heads_kv
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    return torch.softmax(q @ k.transpose(1, 2) / math.sqrt(layer.head_dim), -1) @ v


def test_training_step_against_autograd():
    """With every block selected the layer is dense attention: in fp32 its gradients are
    autograd's.  Bound: 2^-14 of each gradient's norm (sums of at most 512 tokens and 256
    elements in fp32 through five stages, each off by less than 2^-17 of its result)."""
    from video_layer import Layer
    grid = (8, 8, 8)
    layer = Layer(head_dim=64, axes=(16, 24, 24), top_k=8, dtype=torch.float32)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(1, 512, layer.heads_q * 64, generator=g)
    dout = torch.randn(1, layer.heads_q, 512, 64, generator=g)
    o, dw, dq_gain, dk_gain = layer.training_step(x.cuda(), dout.cuda(), grid)
    w = layer.w_qkv.double().cpu().requires_grad_()
    gains = [t.double().cpu().requires_grad_() for t in (layer.q_gain, layer.k_gain)]
    y = attend(layer, *plain(layer, x.double(), w, gains, grid))
    places = ref.place_of(layer.problem(1, grid, 4))[0]
    want = torch.autograd.grad((y * dout[0][:, places].double()).sum(), [w, *gains])
    for name, a, b in zip(("o", "dw", "dq_gain", "dk_gain"), (o[0][:, places], dw, dq_gain, dk_gain), (y, *want)):
        far = (a.double().cpu() - b).norm() / b.norm()
        assert far <= 2.0 ** -14, (name, float(far))


def test_streaming_against_a_plain_cache():
    """Each chunk attends all tokens so far, whose keys and values are the quantised ones.
    The keys are rounded to bf16 twice on the way (projection, rotation), where the plain
    layer rounds nothing, and a different code is 2^-3 of a value off at most: bound by the
    codes' own rounding, 2^-4 of the output's norm."""
    from video_layer import Layer
    grid, h, w = (5, 6, 9), 6, 9
    layer = Layer(heads_q=6, heads_kv=3)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(1, 5 * h * w, layer.heads_q * 128, generator=g).bfloat16()
    got = list(layer.stream(x.cuda().split([54, 162, 54], 1), grid))
    gains = [t.double().cpu() for t in (layer.q_gain, layer.k_gain)]
    q, k, v = plain(layer, x.double(), layer.w_qkv.double().cpu(), gains, grid)
    k, v = (ref.VALUES[c] * torch.pow(2.0, e.double())[..., None] for c, e in (ref.quantised(k), ref.quantised(v)))
    done = 0
    for y in got:
        n = y.shape[1]
        want = attend(layer, q[:, done:done + n], k[:, :done + n], v[:, :done + n])
        want = want.transpose(0, 1).flatten(1)
        far = (y[0].double().cpu() - want).norm() / want.norm()
        assert far <= 2.0 ** -4, float(far)
        done += n
    assert done == 5 * h * w
