"""Attention over a shared list and each sequence's own, against the plain 64-bit form
on the same codes; the bounds are those of the plain attention (test_gpu_attn_cache.py):
joining pieces rounds once more per piece, which the 2^-19 of W for fp32 sums holds."""
import pytest
import torch

import around_reference as ref
import paging_reference as pref
import paper_2609_32882_amd as vsa2
from test_gpu_attn_cache import DT, check, gpu

pytestmark = pytest.mark.gpu

# groups, samples, hq, hkv, D, n, prefix lengths, own lengths, counts (None: n), causal, lists per head, dtype
CASES = [
    (1, 1, 1, 1, 64, 1, [1], [1], None, False, False, "bf16"),
    (1, 3, 10, 2, 128, 1, [130], [0, 64, 65], None, False, False, "bf16"),
    (2, 2, 2, 1, 128, 1, [64, 0], [63, 0, 5, 0], None, True, False, "f32"),
    (2, 3, 6, 2, 64, 5, [300, 77], [5, 3, 70, 8, 130, 6], [5, 4, 0, 1, 5, 5], True, False, "f32"),
    (1, 20, 8, 2, 64, 1, [600], [7 * i for i in range(20)], None, False, True, "bf16"),
    (3, 1, 4, 4, 128, 16, [65, 0, 200], [16, 40, 100], None, True, False, "bf16"),
    (1, 40, 8, 1, 64, 1, [257], [3 + i for i in range(40)], None, False, False, "bf16"),
    (1, 70, 8, 1, 64, 1, [201], [2 + i % 9 for i in range(70)], None, False, False, "bf16"),  # more than 512 rows
    (1, 19, 3, 1, 128, 10, [65], [12] * 19, None, True, False, "f32"),
    (1, 30, 3, 1, 128, 3, [129], [10] * 30, None, True, False, "f32"),
    (1, 2, 4, 2, 64, 40, [190], [64, 41], [40, 39], True, False, "bf16"),                     # many rows on both sides
    (2, 2, 2, 1, 128, 70, [128, 63], [70, 72, 100, 3], [70, 0, 70, 3], False, False, "bf16"),
    (1, 3, 1, 1, 128, 66, [150], [66, 70, 1], [66, 66, 1], True, False, "f32"),
    (2, 2, 2, 1, 64, 64, [70, 1], [64, 0, 100, 64], [64, 0, 10, 64], False, True, "bf16"),
    (1, 2, 1, 1, 64, 100, [0], [150, 100], None, True, False, "bf16"),                        # nothing shared
    (1, 2, 2, 1, 128, 150, [700], [200, 513], None, True, False, "bf16"),
    (1, 5, 2, 1, 128, 1, [2300], [100, 0, 64, 1, 33], None, False, False, "bf16"),            # a list in many pieces
]
IDS = ["%dx%d-%d/%d-D%d-n%d-%s%s-%s" % (*c[:6], "_".join(map(str, c[6])), "-causal" if c[9] else "", c[11]) for c in CASES]


def make(case, seed=0, spread=1.0):
    """Two pools whose pages hold values at their lists' positions and NaN everywhere else."""
    groups, samples, hq, hkv, D, n, plen, lengths, counts, causal, lists, dtype = case
    g = torch.Generator().manual_seed(seed)
    out = []
    for lens in (plen, lengths):
        m = max(1, -(-max(lens) // 64)) + 1
        pages = len(lens) * m + 2
        pool = torch.full((pages, hkv, 128 * D + 128), 0xff, dtype=torch.uint8)
        table = torch.randperm(pages, generator=g)[:len(lens) * m].to(torch.int32).view(len(lens), m)
        if lists:
            table = torch.stack([table.flatten().roll(h).view(len(lens), m) for h in range(hkv)], 1).contiguous()
        top = max(max(lens), 1)
        k = torch.randn(len(lens), hkv, top, D, generator=g) * spread
        v = torch.randn(len(lens), hkv, top, D, generator=g) * torch.randn(len(lens), hkv, top, 1, generator=g).exp()
        ref.write_reference(pool, table, k, v, [0] * len(lens), lens)
        out += [pool, table, torch.tensor(lens, dtype=torch.int32)]
    q = torch.randn(groups * samples, n, hq, D, generator=g).to(DT[dtype]).transpose(1, 2)
    return (*out, q, None if counts is None else torch.tensor(counts, dtype=torch.int32))


def run(case, x, **kw):
    pp, pt, pl, pool, table, length, q, count = (gpu(t) for t in x)
    return vsa2.attn_cache_shared(vsa2.KVCache(pp, pt), vsa2.KVCache(pool, table), q, pl, length, count, causal=case[9], **kw)


def reference(case, x):
    pp, pt, pl, pool, table, length, q, count = x
    return pref.shared_reference(pp, pt, pool, table, q, pl, length, count, case[9])


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_matches_the_plain_form(case):
    x = make(case)
    got = run(case, x)
    check(got, reference(case, x), case[11])
    again = run(case, x)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("i", [1, 3, 6, 9])
def test_peaked_weights(i):
    x = make(CASES[i], seed=1, spread=12.0)
    check(run(CASES[i], x), reference(CASES[i], x), CASES[i][11])


def test_pages_left_out_and_lengths_cut():
    case = (1, 2, 4, 2, 64, 3, [200], [100, 150], None, False, False, "f32")
    x = list(make(case))
    x[1][0, 1], x[4][0, 0], x[4][1, 2] = -5, x[3].shape[0], 2 ** 31 - 1
    check(run(case, x), reference(case, x), "f32")
    x[2][0], x[5][0], x[5][1] = -1, -2 ** 31, 0
    o, lse = run(case, x)
    assert (o == 0).all() and torch.isneginf(lse).all()
    x = list(make(case))
    want = run(case, x)
    m = [x[1].shape[-1] * 64, x[4].shape[-1] * 64]
    x[2], x[5] = torch.tensor([m[0]]).int(), torch.tensor([m[1]] * 2).int()
    full = run(case, x)
    x[2][0], x[5][:] = 2 ** 31 - 1, 2 ** 31 - 1
    cut = run(case, x)
    # (the positions past the lengths hold NaN: both see them alike)
    assert torch.equal(torch.isnan(full[0]), torch.isnan(cut[0])) and torch.isnan(cut[0]).any() and not torch.isnan(want[0]).any()


@pytest.mark.parametrize("side", [0, 1])
@pytest.mark.parametrize("which", [0, 1])
def test_nan_reaches_only_the_rows_that_see_it(side, which):
    case = (2, 2, 2, 1, 64, 2, [100, 100], [70, 71, 72, 73], None, True, False, "bf16")
    x = list(make(case))
    clean = run(case, x)
    pool, table, lists = x[0 if side == 0 else 3], x[1 if side == 0 else 4], 1
    bad = 99 if side == 0 else 70             # the second group's, or its own second sequence's last
    pos = bad if side == 0 else 70
    pool[ref.page_for(table, lists, 0, pos, pool.shape[0]), 0, ref.offsets(pos % 64, 64)[which][5]] = 0x7f
    o, lse = (t.cpu() for t in run(case, x))
    hit = torch.zeros(4, 2, 2, dtype=torch.bool)
    if side == 0:
        hit[2:] = True
    else:
        hit[1, :, 1] = True
    nan = torch.isnan(o)
    assert torch.equal(o[~hit], clean[0].cpu()[~hit]) and not nan[~hit].any()
    assert nan[hit].all() if which == 0 else (nan[hit].sum(-1) == 1).all() and nan[hit][:, 5].all()
    assert torch.equal(torch.isnan(lse), hit if which == 0 else torch.zeros_like(hit))


def test_layouts_streams_guards_and_workspace():
    case = CASES[3]
    x = make(case)
    got = run(case, x)
    groups, samples, hq, hkv, D, n = case[:6]
    batch = groups * samples
    buf = torch.full((batch, n + 2, hq + 2, D), 7.0, device="cuda")
    o = buf[:, 1:-1, 1:-1].transpose(1, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, lse2 = run(case, (*x[:6], x[6].contiguous(), x[7]), o=o)
    side.synchronize()
    assert o2 is o and torch.equal(o, got[0]) and torch.equal(lse2, got[1])
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[:, 1:-1, 1:-1] = True
    assert (buf[~inside] == 7).all()
    none = run(case, (*x[:6], x[6][:, :, :0], x[7]))
    assert none[0].shape == (batch, hq, 0, D) and none[1].shape == (batch, hq, 0)
    # the workspace between guards
    pp, pt, pl, pool, table, length, q, count = (gpu(t) for t in x)
    pre, cache = vsa2.KVCache(pp, pt), vsa2.KVCache(pool, table)
    st, need = vsa2.vsa2_attn_cache_shared_workspace(pre.c, cache.c, hq, n)
    assert st == 0
    ws = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(batch, hq, n, D, device="cuda"), torch.empty(batch, hq, n, device="cuda")
    rows = [vsa2.vsa2_rows(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)) for t in (q, out)]
    st = vsa2.vsa2_attn_cache_shared(pre.c, cache.c, vsa2.VSA2_F32, hq, n, rows[0], pl.data_ptr(), length.data_ptr(),
                                     count.data_ptr(), 1, rows[1], lse.data_ptr(), ws.data_ptr() + 256, need,
                                     torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
    assert (ws[:256] == 0xa5).all() and (ws[256 + need:] == 0xa5).all()


def test_replayed_in_a_graph():
    case = (1, 4, 8, 2, 128, 1, [900], [300, 10, 64, 200], None, False, False, "bf16")
    x = make(case)
    pp, pt, pl, pool, table, length, q, _ = (gpu(t) for t in x)
    pre, cache = vsa2.KVCache(pp, pt), vsa2.KVCache(pool, table)
    step = lambda: vsa2.attn_cache_shared(pre, cache, q, pl, length)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)))
        pl.fill_(300 + 97 * seed)
        length.fill_(10 + seed)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):           # (the second sequence sees NaN from its eleventh token on)
            bits = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
            assert torch.equal(a.view(bits), b.view(bits))
