"""Attention over the 8-bit cache with capped scores, a bias by distance, windows
and spans, against the plain 64-bit form on the same codes.

Bounds: those of the plain attention (test_gpu_attn_cache.py) with the options' part of a
logit's error.  tanh's slope is at most one, so the product's error stays what it is.
cap tanh(y) itself: the exponent's argument has three roundings (3 2^-24 of 2 |y|, which
tanh's slope turns into 0.45 of that at most), exp2 and the reciprocal one unit each, the
last product one: below 2^-21 of cap.  slope |p - j|: the slope's product with log2 e, the
distance and the sum are rounded once each: below 2^-21 of the largest distance times the
slope."""
import pytest
import torch

import around_reference as ref
import paging_reference as pref
import paper_2609_32882_amd as vsa2
from test_gpu_attn_cache import DT, gpu, make

pytestmark = pytest.mark.gpu

# the case of test_gpu_attn_cache (batch, hq, hkv, D, n, max_pages, lengths, counts, causal, lists per head, dtype),
# then cap, slope, window, sink, span ("doc": the token's document of 150, "holes": ends anywhere, None)
CASES = [
    ((1, 1, 1, 64, 1, 1, [1], None, False, False, "bf16"), 30.0, True, 0, 0, None),
    ((3, 10, 2, 128, 1, 9, [0, 65, 570], None, False, False, "bf16"), 30.0, False, 0, 0, None),
    ((3, 10, 2, 128, 1, 9, [1, 130, 570], None, True, False, "f32"), 5.0, True, 64, 3, None),
    ((2, 6, 2, 64, 1, 12, [700, 641], None, False, True, "bf16"), 0.0, True, 200, 70, None),
    ((2, 6, 2, 64, 5, 5, [3, 300], [5, 4], True, False, "f32"), 50.0, True, 17, 0, "doc"),
    ((2, 4, 2, 64, 7, 5, [320, 300], None, False, False, "bf16"), 0.0, False, 0, 0, "holes"),
    ((1, 8, 1, 128, 9, 4, [201], None, False, False, "f32"), 20.0, False, 1, 1, None),
    ((1, 4, 1, 128, 16, 10, [610], None, True, False, "bf16"), 30.0, True, 90, 64, "doc"),
    ((2, 4, 2, 128, 20, 6, [384, 333], [20, 0], False, False, "bf16"), 15.0, True, 0, 5, "holes"),
    ((1, 2, 2, 64, 30, 8, [500], None, True, False, "f32"), 10.0, True, 128, 128, "holes"),
    ((1, 2, 1, 128, 70, 5, [320], None, True, False, "bf16"), 30.0, True, 100, 4, None),
    ((2, 2, 1, 64, 130, 4, [250, 130], [130, 77], True, False, "bf16"), 0.0, True, 65, 1, "doc"),
    ((1, 2, 1, 128, 65, 6, [370], None, False, False, "f32"), 50.0, True, 0, 0, "holes"),
    ((1, 1, 1, 64, 200, 12, [760], None, True, False, "bf16"), 30.0, False, 150, 130, None),
    ((1, 1, 1, 64, 140, 9, [560], None, False, False, "f32"), 0.0, True, 190, 0, "holes"),
    ((1, 3, 3, 128, 1, 30, [1900], None, False, False, "bf16"), 30.0, False, 1500, 4, None),    # several pieces
]
IDS = ["%dx%d/%d-D%d-n%d-%s-%s-cap%g%s-w%d-s%d-%s" % (*c[:5], "_".join(map(str, c[6])), c[10], cap, "-slope" if sl else "", w,
                                                      s, sp) for c, cap, sl, w, s, sp in CASES]


def options(case, cap, slope, window, sink, span, seed=0):
    """The options' tensors (CPU)."""
    batch, hq, n, lengths, counts = case[0], case[1], case[4], case[6], case[7]
    g = torch.Generator().manual_seed(100 + seed)
    out = dict(cap=cap, window=window, sink=sink, slope=None, span=None)
    if slope:
        out["slope"] = (torch.rand(hq, generator=g) - 0.2) * 0.05
    if span:
        at = torch.tensor(lengths)[:, None] - torch.tensor(counts or [n] * batch)[:, None] + torch.arange(n)
        if span == "doc":
            lo = at.clamp_min(0) // 150 * 150
            hi = lo + 150
        else:
            top = max(lengths)
            lo = torch.randint(-5, top, (batch, n), generator=g)
            hi = lo + torch.randint(-3, top, (batch, n), generator=g)
            lo[:, ::5], hi[:, ::3] = -2 ** 31, 2 ** 31 - 1
            lo[:, 1::7] = 2 ** 31 - 1
            hi[:, 2::7] = -2 ** 31
        out["span"] = torch.stack([lo, hi], -1).to(torch.int32)
    return out


def seen(case, opt):
    """bool [batch, n, positions]: what each token sees, by the definition."""
    batch, n, m, lengths, counts, causal = case[0], case[4], case[5], case[6], case[7], case[8]
    j = torch.arange(m * 64)
    out = torch.zeros(batch, n, m * 64, dtype=torch.bool)
    for b in range(batch):
        cnt = n if counts is None else counts[b]
        for i in range(cnt):
            p = lengths[b] - cnt + i
            near = torch.ones_like(j, dtype=torch.bool)
            if opt["window"]:
                near &= j > p - opt["window"]
            if opt["span"] is not None:
                near &= (j >= opt["span"][b, i, 0]) & (j < opt["span"][b, i, 1])
            out[b, i] = ((j < opt["sink"]) | near) & (j < (p + 1 if causal else lengths[b]))
    return out


def poisoned(case, x, opt):
    """The pool with every position that no token sees all ones (codes NaN, powers 2^128)."""
    pool, table = x[0].clone(), x[1]
    some, D = seen(case, opt).any(1), case[3]
    for b in range(case[0]):
        for pos in (~some[b]).nonzero().flatten().tolist():
            for h in range(case[2]):
                page = ref.page_for(table, b, h, pos, pool.shape[0])
                for at in ref.offsets(pos % 64, D):
                    pool[page, h, at] = 0xff
    return pool


def run(case, pool, x, opt, **kw):
    o = {k: (v.cuda() if torch.is_tensor(v) else v) for k, v in opt.items()}
    return vsa2.attn_cache_scored(vsa2.KVCache(pool.cuda(), x[1].cuda()), x[2].cuda(), x[3].cuda(), gpu(x[4]), causal=case[8],
                                  **o, **kw)


def check(got, want, case, opt):
    o, lse = (x.double().cpu() for x in got)
    wo, wl, weight, logit = want
    far = max(max(case[6]), case[4]) * (opt["slope"].double().abs().max() if opt["slope"] is not None else 0.0)
    delta = 2.0 ** -20 * logit + 2.0 ** -21 * (1 + opt["cap"] + far)
    if case[10] == "bf16":
        bound = 2.0 ** -8 * (1 + 2.0 ** -6) * wo.abs() + (2.0 ** -8 + 2 * delta + 2.0 ** -19) * weight
    else:
        bound = (2 * delta + 2.0 ** -19) * weight
    assert ((o - wo).abs() <= bound).all(), ((o - wo).abs() - bound).max()
    empty = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all()
    assert (o[empty] == 0).all()
    lb = delta[..., 0] + 2.0 ** -21 * (1 + wl.abs())
    assert ((lse - wl).abs()[~empty] <= lb[~empty]).all()


@pytest.mark.parametrize("case,cap,slope,window,sink,span", CASES, ids=IDS)
def test_matches_the_plain_form(case, cap, slope, window, sink, span):
    x = make(case)
    opt = options(case, cap, slope, window, sink, span)
    pool = poisoned(case, x, opt)
    got = run(case, pool, x, opt)
    check(got, pref.scored_reference(pool, x[1], x[2], x[3], x[4], case[8], **opt), case, opt)
    again = run(case, pool, x, opt)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("i", [1, 4, 10, 12])
def test_peaked_weights(i):
    """Logits of some tens, far into the cap."""
    case, opt = CASES[i][0], options(CASES[i][0], *CASES[i][1:], seed=1)
    x = make(case, seed=1, spread=12.0)
    check(run(case, x[0], x, opt), pref.scored_reference(*x[:5], case[8], **opt), case, opt)


@pytest.mark.parametrize("i", [1, 6, 12])
def test_without_options_it_is_the_plain_attention(i):
    """Same positions, same scores: the plain attention's own bounds hold for the difference."""
    case = CASES[i][0]
    x = make(case)
    opt = dict(cap=0.0, slope=None, window=0, sink=0, span=None)
    check(run(case, x[0], x, opt), ref.attn_reference(*x[:3], x[3], x[4], case[8]), case, opt)


@pytest.mark.parametrize("n", [3, 130])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [0.0, 2.0 ** -20, 2.0 ** 20])
def test_slopes_and_caps_at_their_ends(n, dtype, cap):
    """A slope of 2^90 leaves the token itself, its weight 1 and its score the lse; -2^90 the list's first."""
    case = (2, 4, 2, 64, n, 5, [290, 201], None, True, False, dtype)
    x = make(case)
    opt = dict(cap=cap, slope=torch.tensor([2.0 ** 90, -2.0 ** 90, 2.0 ** 90, 0.0]), window=0, sink=0, span=None)
    o, lse = (y.double().cpu() for y in run(case, x[0], x, opt))
    wo, wl, weight, logit = pref.scored_reference(*x[:5], case[8], **opt)
    # one term: the weight's fp16 (2^-11) and the result's rounding, or three bf16 terms of the weight, their
    # products' sum, the reciprocal and its product, some 2^-24 each
    step = 2.0 ** -8 + 2.0 ** -10 if dtype == "bf16" else 2.0 ** -21
    assert ((o - wo).abs()[:, :3] <= step * wo.abs()[:, :3]).all()
    # own scores: the product's error and that of log2 e and back; far ones: the distance's product
    delta = 2.0 ** -20 * logit[..., 0] + 2.0 ** -21 * (1 + wl.abs() + min(cap, 64.0))
    assert ((lse - wl).abs() <= delta).all()
    # without a slope the cap alone (errors as in check)
    bound = step * wo.abs() + ((2.0 ** -8 if dtype == "bf16" else 0) + 2 * delta[..., None] + 2.0 ** -19) * weight
    assert ((o - wo).abs() <= bound)[:, 3].all()


@pytest.mark.parametrize("n", [3, 130])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_scores_beside_large_ones(n, dtype):
    """A token whose scores pass half of a large cap takes no bits from the others of its tile."""
    case = (1, 2, 1, 64, n, 5, [290], None, False, False, dtype)
    x = make(case)
    x[2][:, :, 0] *= 2.0 ** 14
    opt = dict(cap=2.0 ** 14, slope=None, window=0, sink=0, span=None)
    o, lse = (y.double().cpu() for y in run(case, x[0], x, opt))
    wo, wl, weight, logit = pref.scored_reference(*x[:5], case[8], **opt)
    delta = 2.0 ** -20 * logit + 2.0 ** -21             # without a part of the cap: the polynomial's is relative
    bound = (2.0 ** -8 * (1 + 2.0 ** -6) * wo.abs() if dtype == "bf16" else 0) + (
        (2.0 ** -8 if dtype == "bf16" else 0) + 2 * delta + 2.0 ** -19) * weight
    assert ((o - wo).abs() <= bound)[:, :, 1:].all()
    assert ((lse - wl).abs() <= delta[..., 0] + 2.0 ** -21 * (1 + wl.abs()))[:, :, 1:].all()


@pytest.mark.parametrize("n", [4, 150])
@pytest.mark.parametrize("which", [0, 1])
def test_nan_reaches_only_the_rows_that_see_it(n, which):
    """A NaN key or value token inside the window of some of the call's tokens."""
    case = (1, 1, 1, 64, n, 6, [330], None, True, False, "bf16")
    opt = options(case, 30.0, True, 40, 2, None)
    x = make(case)
    clean = run(case, x[0], x, opt)
    bad = 330 - n // 2
    hit = seen(case, opt)[0, :, bad]
    assert hit.any() and not hit.all()
    pool = x[0].clone()
    pool[ref.page_for(x[1], 0, 0, bad, pool.shape[0]), 0, ref.offsets(bad % 64, 64)[which][5]] = 0x7f
    o, lse = (t.cpu() for t in run(case, pool, x, opt))
    nan = torch.isnan(o[0, 0])
    assert not nan[~hit].any() and torch.equal(o[0, 0][~hit], clean[0].cpu()[0, 0][~hit])
    assert nan[hit].all() if which == 0 else (nan[hit].sum(-1) == 1).all() and nan[hit][:, 5].all()
    assert torch.equal(torch.isnan(lse[0, 0]), hit if which == 0 else torch.zeros_like(hit))


def test_pages_behind_the_window_may_be_gone():
    """Entries of pages that no row sees are never followed, of pages that some row sees left out."""
    case = (2, 4, 2, 64, 3, 8, [500, 512], None, True, False, "f32")
    opt = options(case, 20.0, True, 70, 10, None)
    x = make(case)
    want = run(case, x[0], x, opt)
    table = x[1].clone()
    table[:, 1:5] = torch.tensor([-1, x[0].shape[0], 2 ** 31 - 1, -2 ** 31])
    y = (x[0], table, *x[2:])
    got = run(case, x[0], y, opt)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    table[:, 7] = -1
    check(run(case, x[0], y, opt), pref.scored_reference(*y[:5], case[8], **opt), case, opt)


def test_layouts_streams_and_guards():
    case = CASES[4][0]
    x = make(case)
    opt = options(case, *CASES[4][1:])
    got = run(case, x[0], x, opt)
    batch, hq, _, D, n = case[:5]
    buf = torch.full((batch, n + 2, hq + 2, D), 7.0, device="cuda")
    o = buf[:, 1:-1, 1:-1].transpose(1, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, lse2 = run(case, x[0], (*x[:2], x[2].contiguous(), *x[3:]), opt, o=o)
    side.synchronize()
    assert o2 is o and torch.equal(o, got[0]) and torch.equal(lse2, got[1])
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[:, 1:-1, 1:-1] = True
    assert (buf[~inside] == 7).all()
    none = run(case, x[0], (*x[:2], x[2][:, :, :0], *x[3:]), dict(opt, span=None))
    assert none[0].shape == (batch, hq, 0, D) and none[1].shape == (batch, hq, 0)


def test_replayed_in_a_graph():
    case = (2, 8, 2, 128, 1, 30, [1900, 700], None, False, False, "bf16")
    x = make(case)
    opt = options(case, 30.0, True, 600, 4, None)
    cache = vsa2.KVCache(x[0].cuda(), x[1].cuda())
    q, length, slope = x[2].cuda(), x[3].cuda(), opt["slope"].cuda()

    def step():
        return vsa2.attn_cache_scored(cache, q, length, cap=30.0, slope=slope, window=600, sink=4)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)))
        length.fill_(700 + 97 * seed)
        slope.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):           # (the second sequence sees NaN past its 700 tokens)
            bits = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
            assert torch.equal(a.view(bits), b.view(bits))
