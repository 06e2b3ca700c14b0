"""The ways a call of attention over the 8-bit cache is cut (tiles of 16, 32 and 128
rows, lists in one piece, several or many, pieces spread over the XCDs), against the
plain 64-bit form with the bounds of test_gpu_attn_cache.py, which hold for any cut."""
import math

import pytest
import torch

import around_reference as ref
import paper_2609_32882_amd as vsa2
from test_gpu_attn_cache import DT, check, gpu, run

pytestmark = pytest.mark.gpu


def lens(batch, longest, step):
    return [max(0, longest - step * b) for b in range(batch)]


def counts(batch, n):
    return [n - b % (n + 1) for b in range(batch)]


# batch, hq, hkv, D, n, max_pages, lengths, counts (None: n), causal, lists per head, dtype
CUTS = {
    "pair, one piece": (16, 4, 4, 64, 20, 5, lens(16, 320, 19), counts(16, 20), True, False, "bf16"),
    "pair, one piece, fp32": (16, 4, 4, 64, 20, 5, lens(16, 320, 19), counts(16, 20), False, True, "f32"),
    "pair, one piece, D 128": (17, 8, 4, 128, 15, 3, lens(17, 192, 9), None, False, False, "bf16"),
    "pair, pieces": (16, 8, 4, 64, 16, 128, lens(16, 1100, 70), counts(16, 16), True, False, "bf16"),
    "pair, pieces, fp32": (16, 8, 4, 64, 16, 128, lens(16, 1100, 70), None, True, False, "f32"),
    "pair and a half, pieces": (11, 4, 4, 128, 40, 130, lens(11, 800, 80), counts(11, 40), False, False, "bf16"),
    "many pieces": (1, 2, 1, 64, 1, 200, [12700], None, False, False, "bf16"),
    "many pieces, fp32": (1, 3, 1, 128, 5, 150, [9500], None, True, False, "f32"),
    "long list, one piece": (32, 4, 4, 64, 1, 70, lens(32, 4480, 140), None, False, False, "bf16"),
    "long list, one piece, fp32": (48, 4, 4, 64, 1, 40, lens(48, 2560, 54), counts(48, 1), False, False, "f32"),
    "128 rows, spread": (16, 8, 8, 64, 130, 3, lens(16, 192, 5), counts(16, 130), False, False, "bf16"),
    "128 rows, spread, fp32": (13, 10, 10, 64, 129, 4, lens(13, 256, 17), counts(13, 129), True, False, "f32"),
    "128 rows, D 128, pieces": (3, 2, 2, 128, 140, 17, [1088, 640, 77], [140, 31, 0], False, False, "bf16"),
}


def page_places(D):
    """Byte of every token's K codes, V codes [64, D] and powers [64] in a page."""
    at = ref.offsets(torch.arange(64)[:, None], D)
    return at[0], at[1], at[2][:, 0], at[3][:, 0]


def make(case, seed=0):
    """A pool with finite codes and powers around one at the lists' positions, and NaN
    everywhere else (codes and powers of all ones)."""
    batch, hq, hkv, D, n, max_pages, lengths, count, causal, lists, dtype = case
    g = torch.Generator().manual_seed(seed)
    pages = batch * max_pages + 2
    pool = torch.full((pages, hkv, 128 * D + 128), 0xff, dtype=torch.uint8)
    order = torch.randperm(pages, generator=g)[:batch * max_pages].to(torch.int32)
    table = order.view(batch, max_pages)
    if lists:
        table = torch.stack([order.roll(h).view(batch, max_pages) for h in range(hkv)], 1).contiguous()
    places = page_places(D)
    for b, length in enumerate(lengths):
        for at in range(0, length, 64):
            m = min(64, length - at)
            for h in range(hkv):
                page = ref.page_for(table, b, h, at, pages)
                for x in range(2):
                    codes = torch.randint(0, 120, (m, D), generator=g) | torch.randint(0, 2, (m, D), generator=g) << 7
                    pool[page, h, places[x][:m]] = codes.to(torch.uint8)
                    pool[page, h, places[2 + x][:m]] = torch.randint(119, 123, (m,), generator=g).to(torch.uint8)
    q = torch.randn(batch, n, hq, D, generator=g).to(DT[dtype])
    return (pool, table, q.transpose(1, 2), torch.tensor(lengths, dtype=torch.int32),
            None if count is None else torch.tensor(count, dtype=torch.int32))


def plain(pool, table, q, length, count, causal):
    """ref.attn_reference a list at a time: (o, lse, sum p |v|, largest sum |q k| / sqrt(D))."""
    batch, hq, n, D = q.shape
    hkv = pool.shape[1]
    group, places = hq // hkv, page_places(D)
    o, weight = (torch.zeros(batch, hq, n, D, dtype=torch.float64) for _ in range(2))
    lse = torch.full((batch, hq, n), -math.inf, dtype=torch.float64)
    logit = torch.zeros(batch, hq, n, 1, dtype=torch.float64)
    for b in range(batch):
        total, cnt = int(length[b]), n if count is None else int(count[b])
        i = torch.arange(n)
        limit = torch.where(i < cnt, total - (cnt - 1 - i) if causal else total, 0).clamp_min(0)
        hidden = torch.arange(total) >= limit[:, None]
        some = limit > 0
        if not some.any():
            continue
        for h in range(hkv):
            ids = [ref.page_for(table, b, h, at, pool.shape[0]) for at in range(0, total, 64)]
            rows = pool[ids, h]
            k, v = (ref.VALUES[rows[:, places[x]].long()] * 2.0 ** (rows[:, places[2 + x]].double() - 127)[..., None]
                    for x in range(2))
            k, v = k.flatten(0, 1)[:total], v.flatten(0, 1)[:total]
            for y in range(h * group, (h + 1) * group):
                x = q[b, y, some].double()
                s = (x @ k.t() / math.sqrt(D)).masked_fill(hidden[some], -math.inf)
                w = torch.softmax(s, -1)
                lse[b, y, some] = torch.logsumexp(s, -1)
                o[b, y, some], weight[b, y, some] = w @ v, w @ v.abs()
                size = (x.abs() @ k.abs().t()).masked_fill(hidden[some], 0.0)
                logit[b, y, some] = size.amax(-1, keepdim=True) / math.sqrt(D)
    return o, lse, weight, logit


@pytest.mark.parametrize("name", CUTS)
def test_matches_the_plain_form(name):
    case = CUTS[name]
    x = make(case, seed=3)
    got = run(case, *x)
    check(got, plain(*x, case[8]), case[10])
    again = run(case, *x)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("name", ["pair, one piece", "pair and a half, pieces", "128 rows, spread",
                                  "128 rows, D 128, pieces"])
def test_queries_past_a_count_reach_nothing(name):
    """Rows past a sequence's count hold NaN and share their tiles with rows that count."""
    case = CUTS[name]
    pool, table, q, length, count = make(case, seed=3)
    clean = run(case, pool, table, q, length, count)
    past = torch.arange(case[4]) >= count[:, None]
    q = q.masked_fill(past[:, None, :, None], float("nan"))
    o, lse = run(case, pool, table, q, length, count)
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])
    past = past[:, None].expand(lse.shape).cuda()
    assert (o[past] == 0).all() and torch.isneginf(lse[past]).all()


def test_nan_in_a_pair_of_tiles():
    """A NaN value token reaches the rows of both tiles that see it and no others."""
    case = (16, 4, 4, 64, 32, 4, [200] * 16, None, True, False, "bf16")
    pool, table, q, length, count = make(case)
    clean = run(case, pool, table, q, length, count)
    for back in (2, 20):                               # seen by the last rows of tile 2; by some of tile 1 too
        bad = 200 - back
        spoilt = pool.clone()
        spoilt[ref.page_for(table, 0, 1, bad, pool.shape[0]), 1, ref.offsets(bad % 64, 64)[1][5]] = 0x7f
        o, lse = run(case, spoilt, table, q, length, count)
        hit = torch.isnan(o)
        want = torch.zeros_like(hit)
        want[0, 1, 32 - back:, 5] = True
        assert torch.equal(hit, want) and torch.equal(o[~hit], clean[0][~hit]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("name", ["many pieces, fp32", "128 rows, D 128, pieces", "pair, pieces"])
def test_workspace_is_enough_and_kept_to(name):
    case = CUTS[name]
    pool, table, q, length, count = make(case)
    want = run(case, pool, table, q, length, count)
    cache = vsa2.KVCache(pool.cuda(), table.cuda())
    hq, n = case[1], case[4]
    st, need = vsa2.vsa2_attn_cache_workspace(cache.c, hq, n)
    assert st == 0 and need > 0
    ws = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")      # NaN wherever it is read unwritten
    q, length, count = q.cuda(), length.cuda(), gpu(count)
    o, lse = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    rows = [vsa2.vsa2_rows(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)) for t in (q, o)]
    st = vsa2.vsa2_attn_cache(cache.c, vsa2.VSA2_F32 if case[10] == "f32" else vsa2.VSA2_BF16, hq, n, rows[0],
                              length.data_ptr(), None if count is None else count.data_ptr(), int(case[8]), rows[1],
                              lse.data_ptr(), ws.data_ptr() + 256, need, torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    assert (ws[:256] == 0xff).all() and (ws[256 + need:] == 0xff).all()


def test_tables_of_a_rotation_are_kept():
    """Changing the list of tables afterwards does not change (or free) what the rotation reads."""
    p = vsa2.make_problem(1, 1, 1, 64, 1, 1, 8, 1, 1, 1, 1, 1, 1, vsa2.VSA2_F32)
    tables = [None, None, vsa2.rope_table(8, 64)]
    rope = vsa2.Rope((0, 0, 64), tables)
    x = torch.randn(1, 1, 8, 64, device="cuda")
    want = vsa2.qk_norm_rope(p, x, rope=rope)[0].clone()
    tables[2] = None
    torch.full((8, 32, 2), 7.0, device="cuda")         # takes the memory if it was given back
    assert torch.equal(vsa2.qk_norm_rope(p, x, rope=rope)[0], want)
