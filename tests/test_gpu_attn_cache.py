"""Attention over the 8-bit cache against the plain 64-bit form on the same codes.

Bounds.  A logit is a sum of D exact products in fp32: off by at most
delta = 2^-20 of the largest sum of |q_d k_d| / sqrt(D), plus 2^-21 for the
exponential; that moves a weight by a factor of 1 +- delta, the result by
2 delta of W = sum p |v|.  bf16 probabilities are rounded once (2^-8 of W) and so
is the result (2^-8 of itself); fp32 ones enter as three terms, and what is left
are fp32 sums over the list (2^-19 of W)."""
import pytest
import torch

import around_reference as ref
import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# batch, hq, hkv, D, n, max_pages, lengths, counts (None: n), causal, lists per head, dtype
CASES = [
    (1, 1, 1, 64, 1, 1, [1], None, False, False, "bf16"),
    (2, 2, 1, 128, 1, 1, [64, 63], None, True, False, "f32"),
    (3, 10, 2, 128, 1, 9, [0, 65, 570], None, False, False, "bf16"),
    (2, 40, 8, 128, 1, 7, [448, 129], None, False, True, "bf16"),
    (2, 6, 2, 64, 5, 5, [3, 300], [5, 4], True, False, "f32"),       # rows with nothing to attend
    (1, 4, 4, 64, 16, 3, [150], None, True, False, "bf16"),
    (2, 3, 1, 128, 17, 6, [100, 383], [17, 0], True, True, "f32"),
    (1, 8, 1, 128, 9, 4, [201], None, False, False, "bf16"),
    (1, 2, 2, 128, 70, 5, [320], None, True, False, "bf16"),
    (2, 4, 2, 64, 130, 4, [250, 130], [130, 77], True, False, "bf16"),
    (1, 2, 1, 128, 65, 3, [190], None, False, False, "f32"),
    (1, 3, 3, 128, 1, 40, [2500], None, False, False, "bf16"),       # a list in many pieces
    (1, 2, 1, 64, 200, 20, [1270], None, True, False, "bf16"),
]
IDS = ["%dx%d/%d-D%d-n%d-%s%s%s%s" % (c[0], c[1], c[2], c[3], c[4], "_".join(map(str, c[6])), "-causal" if c[8] else "",
                                     "-lists" if c[9] else "", "-" + c[10]) for c in CASES]


def make(case, seed=0, spread=1.0):
    """A pool whose pages hold values written at their list positions and NaN
    everywhere else (codes and powers of all ones)."""
    batch, hq, hkv, D, n, max_pages, lengths, counts, causal, lists, dtype = case
    g = torch.Generator().manual_seed(seed)
    pages = batch * max_pages + 2
    pool = torch.full((pages, hkv, 128 * D + 128), 0xff, dtype=torch.uint8)
    order = torch.randperm(pages, generator=g)[:batch * max_pages].to(torch.int32)
    table = order.view(batch, max_pages)
    if lists:
        table = torch.stack([order.roll(h).view(batch, max_pages) for h in range(hkv)], 1).contiguous()
    m = max(max(lengths), 1)
    k = torch.randn(batch, hkv, m, D, generator=g) * spread
    v = torch.randn(batch, hkv, m, D, generator=g) * torch.randn(batch, hkv, m, 1, generator=g).exp()
    ref.write_reference(pool, table, k, v, [0] * batch, lengths)
    q = torch.randn(batch, n, hq, D, generator=g).to(DT[dtype])
    return (pool, table, q.transpose(1, 2), torch.tensor(lengths, dtype=torch.int32),
            None if counts is None else torch.tensor(counts, dtype=torch.int32))


def gpu(t):
    return None if t is None else t.cuda()


def check(got, want, dtype):
    o, lse = (x.double().cpu() for x in got)
    wo, wl, weight, logit = want
    delta = 2.0 ** -20 * logit + 2.0 ** -21
    if dtype == "bf16":
        bound = 2.0 ** -8 * (1 + 2.0 ** -6) * wo.abs() + (2.0 ** -8 + 2 * delta + 2.0 ** -19) * weight
    else:
        bound = (2 * delta + 2.0 ** -19) * weight
    assert ((o - wo).abs() <= bound).all(), ((o - wo).abs() - bound).max()
    empty = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all()
    assert (o[empty] == 0).all()
    lb = delta[..., 0] + 2.0 ** -21 * (1 + wl.abs())
    assert ((lse - wl).abs()[~empty] <= lb[~empty]).all()


def run(case, pool, table, q, length, count, **kw):
    return vsa2.attn_cache(vsa2.KVCache(pool.cuda(), table.cuda()), q.cuda(), length.cuda(), gpu(count),
                           causal=case[8], **kw)


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_matches_the_plain_form(case):
    x = make(case)
    got = run(case, *x)
    check(got, ref.attn_reference(*x[:3], x[3], x[4], case[8]), case[10])
    again = run(case, *x)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("case", [CASES[2], CASES[6], CASES[8]], ids=[IDS[2], IDS[6], IDS[8]])
def test_peaked_weights(case):
    """Logits of some tens: nearly all weight on few tokens."""
    x = make(case, seed=1, spread=12.0)
    check(run(case, *x), ref.attn_reference(*x[:3], x[3], x[4], case[8]), case[10])


def test_pages_left_out():
    """Entries outside the pool leave their 64 positions out."""
    case = (2, 4, 2, 64, 3, 6, [380, 300], None, False, False, "f32")
    pool, table, q, length, count = make(case)
    table[0, 2], table[0, 5], table[1, 0] = -5, pool.shape[0], 2 ** 31 - 1
    check(run(case, pool, table, q, length, count), ref.attn_reference(pool, table, q, length, count, False), "f32")
    table[:] = -1                                      # nothing at all
    o, lse = run(case, pool, table, q, length, count)
    assert (o == 0).all() and torch.isneginf(lse).all()


def test_lengths_beyond_the_list_are_cut():
    case = (2, 2, 1, 64, 2, 2, [128, 128], None, False, False, "f32")
    pool, table, q, length, count = make(case)
    cut = run(case, pool, table, q, torch.tensor([2 ** 31 - 1, -7], dtype=torch.int32), count)
    full = run(case, pool, table, q, length, count)
    assert torch.equal(cut[0][0], full[0][0]) and (cut[0][1] == 0).all() and torch.isneginf(cut[1][1]).all()


@pytest.mark.parametrize("n", [4, 70])
def test_nan_reaches_only_the_rows_that_see_it(n):
    """A NaN key or value token: rows past it are NaN, rows masked from it are not."""
    case = (1, 2, 1, 64, n, 4, [200], None, True, False, "bf16")
    for which in range(2):
        pool, table, q, length, count = make(case)
        clean = run(case, pool, table, q, length, count)
        bad = 200 - 2                                  # the last but one token
        at = ref.offsets(bad % 64, 64)[which]
        page = ref.page_for(table, 0, 0, bad, pool.shape[0])
        pool[page, 0, at[5]] = 0x7f
        o, lse = run(case, pool, table, q, length, count)
        hit = torch.isnan(o)
        assert not hit[:, :, :n - 2].any() and torch.equal(o[:, :, :n - 2], clean[0][:, :, :n - 2])
        assert hit[:, :, n - 2:, 5].all()
        if which == 0:
            assert hit[:, :, n - 2:].all() and torch.isnan(lse[:, :, n - 2:]).all()
        else:
            assert hit[:, :, n - 2:].sum() == 2 * 2 and not torch.isnan(lse).any()


def test_layouts_streams_and_guards():
    case = CASES[6]
    x = make(case)
    got = run(case, *x)
    batch, hq, _, D, n = case[:5]
    buf = torch.full((batch, n + 2, hq + 2, D), 7.0, device="cuda")
    o = buf[:, 1:-1, 1:-1].transpose(1, 2)
    cache = vsa2.KVCache(x[0].cuda(), x[1].cuda())
    q, length, count = x[2].contiguous().cuda(), x[3].cuda(), gpu(x[4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, lse2 = vsa2.attn_cache(cache, q, length, count, causal=True, o=o)
    side.synchronize()
    assert o2 is o and torch.equal(o, got[0]) and torch.equal(lse2, got[1])
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[:, 1:-1, 1:-1] = True
    assert (buf[~inside] == 7).all()
    none = vsa2.attn_cache(cache, q[:, :, :0], length)
    assert none[0].shape == (batch, hq, 0, D) and none[1].shape == (batch, hq, 0)


@pytest.mark.parametrize("case", [CASES[11], CASES[8]], ids=[IDS[11], IDS[8]])
def test_workspace_is_enough_and_kept_to(case):
    pool, table, q, length, count = make(case)
    cache = vsa2.KVCache(pool.cuda(), table.cuda())
    want = vsa2.attn_cache(cache, q.cuda(), length.cuda(), gpu(count), causal=case[8])
    hq, n = case[1], case[4]
    st, need = vsa2.vsa2_attn_cache_workspace(cache.c, hq, n)
    assert st == 0
    ws = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device="cuda")
    qd = q.cuda()
    o = torch.empty(qd.shape, dtype=qd.dtype, device="cuda")
    lse = torch.empty(qd.shape[:3], device="cuda")
    ln, ct = length.cuda(), gpu(count)
    rows = [vsa2.vsa2_rows(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)) for t in (qd, o)]
    st = vsa2.vsa2_attn_cache(cache.c, vsa2.VSA2_BF16, hq, n, rows[0], ln.data_ptr(), None if ct is None else ct.data_ptr(),
                              int(case[8]), rows[1], lse.data_ptr(), ws.data_ptr() + 256, need,
                              torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    assert (ws[:256] == 0xa5).all() and (ws[256 + need:] == 0xa5).all()


def test_page_addresses_past_four_gigabytes():
    """Pages whose bytes lie past 32 bits."""
    D, hkv = 128, 8
    page = 128 * D + 128
    pages = (1 << 32) // (hkv * page) + 8
    pool = torch.empty(pages, hkv, page, dtype=torch.uint8, device="cuda")
    g = torch.Generator().manual_seed(4)
    k = torch.randn(1, hkv, 100, D, generator=g).cuda()
    q = torch.randn(1, hkv, 1, D, generator=g).bfloat16().cuda()
    start, length = torch.zeros(1, dtype=torch.int32).cuda(), torch.full((1,), 100, dtype=torch.int32).cuda()
    out = []
    for table in ([pages - 1, pages - 4], [0, 1]):
        cache = vsa2.KVCache(pool, torch.tensor([table], dtype=torch.int32).cuda())
        vsa2.cache_write(cache, k, k, start)
        out.append((*vsa2.attn_cache(cache, q, length), *vsa2.cache_read(cache, 100, start)))
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_replayed_in_a_graph():
    case = (2, 8, 2, 128, 1, 30, [1900, 700], None, False, False, "bf16")
    pool, table, q, length, count = make(case)
    cache = vsa2.KVCache(pool.cuda(), table.cuda())
    q, length, start = q.cuda(), length.cuda(), (length - 1).cuda()
    kv = torch.randn(2, 2, 1, 128, device="cuda").bfloat16()

    def step():
        vsa2.cache_write(cache, kv, kv, start)
        return vsa2.attn_cache(cache, q, length)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        kv.copy_(torch.randn(kv.shape, generator=torch.Generator().manual_seed(seed)))
        length.fill_(300 + 97 * seed)
        start.fill_(299 + 97 * seed)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)
