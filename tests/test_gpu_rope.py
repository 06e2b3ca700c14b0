"""vsa2_qk_norm_rope and its gradients against the plain 64-bit form.

Bounds.  The kernels work in fp32: the mean of squares is a sum of D terms in a
tree (relative error below 16 * 2^-24), the reciprocal root adds one ulp, and a
turned element is two products of values with such errors, so an element is off
by at most 2^-20 of |a| + |b| of its pair; a bf16 result is then rounded once
(2^-8 of itself, the unit roundoff of 8 significant bits).  A gradient's row mean adds the same again for the sizes
behind it (2^-19).  A gain's gradient is a sum of at most 64 terms in a row and
a tree: 2^-17 of the sum of sizes."""
import pytest
import torch

import around_reference as ref
import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

EPS = 1e-6
AXES = {64: [(16, 24, 24), (20, 22, 22), (8, 0, 16), (64, 0, 0)],
        128: [(44, 42, 42), (16, 56, 56), (32, 32, 32), (0, 64, 64)]}
# batch, hq, hkv, D, (T, H, W), cube, text, dtype, norm, halves, origin
SHAPES = [
    (1, 2, 2, 64, (1, 1, 1), 1, 0, "f32", True, False, True),
    (1, 1, 1, 128, (1, 1, 1), 4, 0, "bf16", True, False, False),
    (5, 10, 2, 128, (1, 1, 3), 1, 0, "bf16", True, True, True),
    (2, 3, 1, 64, (5, 6, 7), 4, 0, "f32", True, True, False),
    (2, 6, 2, 128, (4, 8, 8), 4, 0, "bf16", True, False, False),
    (1, 4, 4, 128, (3, 9, 5), 4, 70, "f32", True, False, True),
    (1, 8, 1, 64, (9, 4, 4), 4, 1, "bf16", True, True, False),
    (2, 2, 1, 128, (2, 5, 3), 4, 64, "bf16", False, True, True),
    (1, 3, 3, 64, (6, 3, 10), 2, 9, "f32", False, False, False),
    (3, 5, 5, 64, (7, 13, 1), 4, 0, "bf16", True, False, False),
]
IDS = ["%dx%d/%d-D%d-%s-c%d-t%d-%s%s%s%s" % (s[0], s[1], s[2], s[3], "x".join(map(str, s[4])), s[5], s[6], s[7],
                                            "-norm" if s[8] else "", "-halves" if s[9] else "",
                                            "-origin" if s[10] else "") for s in SHAPES]


def make(shape, seed=0, axes_pick=0):
    batch, hq, hkv, D, grid, cube, text, dtype, norm, halves, origin = shape
    g = torch.Generator().manual_seed(100 + seed)
    p = vsa2.make_problem(batch, hq, hkv, D, *grid, cube, cube, cube, 1, 1, 1,
                          vsa2.VSA2_F32 if dtype == "f32" else vsa2.VSA2_BF16, text)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    axes = AXES[D][axes_pick]
    if halves and sum(axes) % 8:
        axes = (16, 24, 24)
    n = grid[0] * grid[1] * grid[2] + text
    x = (torch.randn(batch, n, hq + 2 * hkv, D, generator=g) * torch.randn(1, 1, hq + 2 * hkv, D, generator=g).exp()).to(dt)
    gains = [1 + 0.3 * torch.randn(D, generator=g) for _ in range(2)] if norm else [None, None]
    extra = 9 if origin else 0
    tables = [vsa2.rope_table(m + extra, a, device="cpu") if a else None for m, a in zip(grid, axes)]
    # rows outside the tables (both ends) are clamped
    org = torch.randint(-3, extra + 3, (batch, 3), generator=g, dtype=torch.int32) if origin else None
    return p, dt, x, gains, (EPS if norm else 0.0), axes, tables, org, halves, (hq, hkv)


def rope_on_gpu(axes, tables, org, halves):
    return vsa2.Rope(axes, [None if t is None else t.cuda() for t in tables], None if org is None else org.cuda(),
                     "halves" if halves else "adjacent")


def parts(x, hq, hkv):
    return [y.transpose(1, 2) for y in x.split([hq, hkv, hkv], 2)]


def gpu(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("pick", [0, 2])
def test_forward(shape, pick):
    p, dt, x, gains, eps, axes, tables, org, halves, heads = make(shape, axes_pick=pick)
    places, where, L = ref.place_of(p)
    cs = ref.turn_of(p, axes, tables, org, where)
    out = vsa2.qk_norm_rope(p, *parts(x.cuda(), *heads), q_gain=gpu(gains[0]), k_gain=gpu(gains[1]),
                            rope=rope_on_gpu(axes, tables, org, halves), eps=eps)
    for i, (y, part) in enumerate(zip(out, parts(x, *heads))):
        part = part.double()
        if i < 2:
            want, size = ref.rope_forward(p, part, None if gains[i] is None else gains[i].double(), eps, cs, halves)
        else:
            want, size = part, torch.zeros_like(part)
        want, size = ref.to_places(want, places, L), ref.to_places(size, places, L)
        bound = 2.0 ** -20 * size + (2.0 ** -8 * (1 + 2.0 ** -6) * want.abs() if dt == torch.bfloat16 and i < 2 else 0)
        got = y.double().cpu()
        assert got.shape == want.shape
        assert ((got - want).abs() <= bound).all(), (i, ((got - want).abs() - bound).max())
        real = torch.zeros(L, dtype=torch.bool)
        real[places] = True
        assert (got[:, :, ~real] == 0).all()          # padding


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_backward(shape):
    p, dt, x, gains, eps, axes, tables, org, halves, (hq, hkv) = make(shape, seed=1)
    places, where, L = ref.place_of(p)
    cs = ref.turn_of(p, axes, tables, org, where)
    g = torch.Generator().manual_seed(7)
    dy = [torch.randn(p.batch, h, L, p.head_dim, generator=g).to(dt) for h in (hq, hkv, hkv)]
    for y in dy:                                       # padding must not be looked at
        mask = torch.ones(L, dtype=torch.bool)
        mask[places] = False
        y[:, :, mask] = float("nan")
    q, k, _ = parts(x.cuda(), hq, hkv)
    out = torch.full_like(x, float("nan")).cuda()
    args = dict(q=q, k=k, q_gain=gpu(gains[0]), k_gain=gpu(gains[1]), eps=eps) if eps else {}
    got = vsa2.qk_norm_rope_bwd(p, *(t.cuda() for t in dy), rope=rope_on_gpu(axes, tables, org, halves),
                                out=parts(out, hq, hkv), **args)
    again = vsa2.qk_norm_rope_bwd(p, *(t.cuda() for t in dy), rope=rope_on_gpu(axes, tables, org, halves), **args)
    for i, part in enumerate(parts(x, hq, hkv)):
        d = dy[i][:, :, places].double()
        if i < 2:
            want, dgain, size, gsize = ref.rope_backward(
                part.double(), None if gains[i] is None else gains[i].double(), eps, cs, halves, d)
        else:
            want, dgain, size = d, None, torch.zeros_like(d)
        bound = 2.0 ** -19 * size + (2.0 ** -8 * (1 + 2.0 ** -6) * want.abs() if dt == torch.bfloat16 and i < 2 else 0)
        err = (got[i].double().cpu() - want).abs()
        assert (err <= bound).all(), (i, (err - bound).max())
        assert torch.equal(got[i].cpu(), again[i].cpu())
        if dgain is not None:
            assert ((got[3 + i].double().cpu() - dgain).abs() <= 2.0 ** -17 * gsize).all(), i
            assert torch.equal(got[3 + i], again[3 + i])
        elif i < 2:
            assert got[3 + i] is None


def test_backward_of_many_tokens_sums_the_gains():
    """More token groups than workgroups, so each workgroup takes several."""
    p = vsa2.make_problem(1, 2, 1, 128, 12, 40, 40, 4, 4, 4, 1, 1, 1, vsa2.VSA2_BF16)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = 12 * 40 * 40
    x = torch.randn(1, n, 4, 128, generator=g, device="cuda").bfloat16()
    dy = [torch.randn(1, h, n, 128, generator=g, device="cuda").bfloat16() for h in (2, 1, 1)]
    q, k, _ = parts(x, 2, 1)
    got = vsa2.qk_norm_rope_bwd(p, *dy, q=q, k=k, eps=EPS)
    places = ref.place_of(p)[0].cuda()
    for i, part in enumerate((q, k)):
        d = dy[i][:, :, places].double()
        part = part.double()
        rms = torch.sqrt((part * part).mean(-1, keepdim=True) + EPS)
        want, size = (d * part / rms).sum((0, 1, 2)), (d * part / rms).abs().sum((0, 1, 2))
        # 19,200 tokens of 2 heads in chains of at most 64 per lane, 128 partial rows per adder
        assert ((got[3 + i].double() - want).abs() <= 2.0 ** -16 * size).all()
        assert torch.equal(got[3 + i], vsa2.qk_norm_rope_bwd(p, *dy, q=q, k=k, eps=EPS)[3 + i])


def test_parts_layouts_and_streams():
    """Parts alone give what they give together; rows laid out [batch, heads,
    tokens, D], shared between sequences, and on another stream."""
    shape = SHAPES[5]
    p, dt, x, gains, eps, axes, tables, org, halves, (hq, hkv) = make(shape)
    rope = rope_on_gpu(axes, tables, org, halves)
    q, k, v = parts(x.cuda(), hq, hkv)
    kw = dict(rope=rope, eps=eps)
    all3 = vsa2.qk_norm_rope(p, q, k, v, q_gain=gpu(gains[0]), k_gain=gpu(gains[1]), **kw)
    only_k = vsa2.qk_norm_rope(p, k=k, k_gain=gpu(gains[1]), **kw)
    assert only_k[0] is None and only_k[2] is None and torch.equal(only_k[1], all3[1])
    qc = q.contiguous()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = vsa2.qk_norm_rope(p, qc, q_gain=gpu(gains[0]), **kw)[0]
    side.synchronize()
    assert torch.equal(other, all3[0])
    p2 = vsa2.make_problem(3, hq, hkv, p.head_dim, p.T, p.H, p.W, 4, 4, 4, 1, 1, 1, vsa2.VSA2_F32, p.text_len)
    rope2 = rope_on_gpu(axes, tables, None, halves)
    shared = vsa2.qk_norm_rope(p2, q[:1].expand(3, -1, -1, -1), q_gain=gpu(gains[0]), rope=rope2, eps=eps)[0]
    one = vsa2.qk_norm_rope(p, q, q_gain=gpu(gains[0]), rope=rope2, eps=eps)[0]
    for b in range(3):
        assert torch.equal(shared[b], one[0])


def test_special_rows():
    """A row of zeros stays zero, NaN and infinity stay in their row."""
    p = vsa2.make_problem(1, 2, 2, 64, 1, 4, 4, 4, 4, 4, 1, 1, 1, vsa2.VSA2_F32)
    x = torch.randn(1, 2, 16, 64, generator=torch.Generator().manual_seed(2))
    x[0, 0, 3] = 0
    x[0, 0, 5, 7] = float("nan")
    x[0, 1, 6, 9] = float("inf")
    y = vsa2.qk_norm_rope(p, x.cuda(), eps=EPS)[0].cpu()
    places = ref.place_of(p)[0]
    y = y[:, :, places]
    assert (y[0, 0, 3] == 0).all() and torch.isnan(y[0, 0, 5]).all() and torch.isnan(y[0, 1, 6]).any()
    rest = torch.ones(2, 16, dtype=torch.bool)
    rest[0, 5] = rest[1, 6] = False
    assert torch.isfinite(y[0][rest]).all()


def test_no_write_outside_the_outputs():
    """Guard bytes around every output and the workspace stay as they were."""
    shape = SHAPES[6]
    p, dt, x, gains, eps, axes, tables, org, halves, (hq, hkv) = make(shape)
    rope = rope_on_gpu(axes, tables, org, halves)
    L, D, n = ref.place_of(p)[2], p.head_dim, x.shape[1]
    q, k, v = parts(x.cuda(), hq, hkv)

    def guarded(shape):
        size = 1
        for m in shape:
            size *= m
        buf = torch.full((size + 512,), 7.0, dtype=dt, device="cuda")
        return buf, buf[256:256 + size].view(shape)

    outs = [guarded((1, h, L, D)) for h in (hq, hkv, hkv)]
    vsa2.qk_norm_rope(p, q, k, v, q_gain=gpu(gains[0]), k_gain=gpu(gains[1]), rope=rope, eps=eps,
                      out=[o[1] for o in outs])
    grads = [guarded((1, n, h, D)) for h in (hq, hkv, hkv)]
    vsa2.qk_norm_rope_bwd(p, *(o[1] for o in outs), q=q, k=k, rope=rope, eps=eps,
                          out=[o[1].transpose(1, 2) for o in grads])
    st, need = vsa2.vsa2_qk_norm_rope_workspace(p)
    assert st == 0
    for buf, view in outs + grads:
        assert (buf[:256] == 7).all() and (buf[256 + view.numel():] == 7).all()


def test_finite_differences_and_adjoint():
    """The forward's change along a direction is the gradient's product with it."""
    shape = (1, 2, 1, 64, (2, 3, 5), 4, 3, "f32", True, True, False)
    p, dt, x, gains, eps, axes, tables, org, halves, (hq, hkv) = make(shape, seed=5)
    x = x / x.abs().max() * 2
    rope = rope_on_gpu(axes, tables, org, halves)
    g = torch.Generator().manual_seed(11)
    kw = dict(rope=rope, eps=eps)
    q = parts(x, hq, hkv)[0].contiguous()
    step, dirq, dirg = 2.0 ** -9, torch.randn(q.shape, generator=g), torch.randn(64, generator=g)
    dy = torch.randn(1, hq, ref.place_of(p)[2], 64, generator=g)

    def value(a):
        y = vsa2.qk_norm_rope(p, (q + a * step * dirq).cuda(), q_gain=(gains[0] + a * step * dirg).cuda(), **kw)[0]
        return (y.double().cpu() * dy.double()).sum()

    slope = (value(1) - value(-1)) / (2 * step)
    d = vsa2.qk_norm_rope_bwd(p, dy.cuda(), q=q.cuda(), q_gain=gains[0].cuda(), **kw)
    want = (d[0].double().cpu() * dirq.double()).sum() + (d[3].double().cpu() * dirg.double()).sum()
    # the difference's third-order term: step^2 / 6 of a third derivative of order one per element, over
    # some 4,000 elements, beside fp32 noise of 2^-22 / step of the same sums
    scale = (d[0].double().cpu().abs() * dirq.double().abs()).sum() + (dy.abs().double().sum())
    assert abs(slope - want) <= scale * (step * step * 4 + 2.0 ** -22 / step)


def test_replayed_in_a_graph():
    shape = SHAPES[4]
    p, dt, x, gains, eps, axes, tables, org, halves, (hq, hkv) = make(shape)
    rope = rope_on_gpu(axes, tables, org, halves)
    xg = x.cuda()
    q, k, v = parts(xg, hq, hkv)
    gq, gk = gpu(gains[0]), gpu(gains[1])
    dy = [torch.randn(2, h, ref.place_of(p)[2], 128, device="cuda").bfloat16() for h in (hq, hkv, hkv)]

    def both():
        return vsa2.qk_norm_rope(p, q, k, v, q_gain=gq, k_gain=gk, rope=rope, eps=eps) + \
            vsa2.qk_norm_rope_bwd(p, *dy, q=q, k=k, q_gain=gq, k_gain=gk, rope=rope, eps=eps)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in range(3):
        xg.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)).to(dt))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, both()):
            assert torch.equal(a, b)
