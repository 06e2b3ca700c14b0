"""Calls of more than 128 rows over the cache (a tile of 128 rows whose waves share the
pages): pages left out, lists of many fetches of the table and of many pieces, logits that
rise along the list.  Against the plain 64-bit form with the bounds of
test_gpu_attn_cache.py, which hold for any cut."""
import math

import pytest
import torch

import paper_2609_32882_amd as vsa2
from test_gpu_attn_cache import DT, check

pytestmark = pytest.mark.gpu


def filled(batch, hkv, D, m, seed=0, rising=False):
    """(cache, k, v [batch, heads, m, D] in 64 bits): m tokens a sequence in a pool that is NaN elsewhere."""
    g = torch.Generator().manual_seed(seed)
    width = -(-m // 64)
    pages = batch * width + 2
    table = torch.randperm(pages, generator=g)[:batch * width].to(torch.int32).view(batch, width).cuda()
    pool = torch.full((pages, hkv, 128 * D + 128), 0xff, dtype=torch.uint8, device="cuda")
    cache = vsa2.KVCache(pool, table)
    k, v = (torch.randn(batch, hkv, m, D, generator=g) for _ in range(2))
    if rising:                                  # logits of some tens, the largest at the end
        k = k * torch.linspace(0.5, 12, m)[:, None]
    start = torch.zeros(batch, dtype=torch.int32, device="cuda")
    vsa2.cache_write(cache, k.cuda(), v.cuda(), start)
    k, v = vsa2.cache_read(cache, m, start, dtype=torch.float32)
    return cache, k.double(), v.double()


def plain(k, v, q, lengths, causal, there=None):
    """(o, lse, sum p |v|, largest sum |q k| / sqrt(D)); there [batch, m]: positions whose page exists."""
    batch, hq, n, D = q.shape
    group = hq // k.shape[1]
    o, weight = (torch.zeros(batch, hq, n, D, dtype=torch.float64) for _ in range(2))
    lse = torch.full((batch, hq, n), -math.inf, dtype=torch.float64)
    logit = torch.zeros(batch, hq, n, 1, dtype=torch.float64)
    for b in range(batch):
        limit = lengths[b] - torch.arange(n - 1, -1, -1, device=q.device) * int(causal)
        shown = torch.arange(k.shape[2], device=q.device) < limit[:, None]
        if there is not None:
            shown = shown & there[b].to(q.device)
        some = shown.any(1)
        if not some.any():
            continue
        hide = ~shown[some]
        for h in range(hq):
            x, kk, vv = q[b, h, some].double(), k[b, h // group], v[b, h // group]
            s = (x @ kk.t() / math.sqrt(D)).masked_fill(hide, -math.inf)
            w = torch.softmax(s, -1)
            at = some.cpu()
            lse[b, h, at] = torch.logsumexp(s, -1).cpu()
            o[b, h, at], weight[b, h, at] = (w @ vv).cpu(), (w @ vv.abs()).cpu()
            size = (x.abs() @ kk.abs().t()).masked_fill(hide, 0.0).amax(-1, keepdim=True)
            logit[b, h, at] = (size / math.sqrt(D)).cpu()
    return o, lse, weight, logit


def queries(batch, hq, n, D, dtype, seed=9):
    return torch.randn(batch, hq, n, D, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def compare(cache, k, v, q, lengths, causal, dtype, there=None):
    got = vsa2.attn_cache(cache, q, i32(lengths), causal=causal)
    check(got, plain(k, v, q, lengths, causal, there), dtype)
    again = vsa2.attn_cache(cache, q, i32(lengths), causal=causal)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
def test_logits_that_rise_along_the_list(D, dtype, causal):
    cache, k, v = filled(2, 2, D, 700, rising=True)
    compare(cache, k, v, queries(2, 4, 90, D, dtype), [700, 333], causal, dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gone", [(0,), (1,), (1, 2), (0, 3, 4, 7), tuple(range(8)), (10,), tuple(range(1, 11)),
                                  tuple(range(11))], ids=str)
def test_pages_left_out(D, dtype, gone):
    """Entries outside the pool at odd and even places, first and last, side by side, whole pieces of them."""
    m = 650                                     # 11 pages, the last one cut
    cache, k, v = filled(2, 2, D, m, seed=2)
    outside = [-1, cache.pool.shape[0], 2 ** 31 - 1, -2 ** 31]
    there = torch.ones(2, m, dtype=torch.bool)
    for x, page in enumerate(gone):             # the second sequence keeps its pages
        cache.table[0, page] = outside[x % 4]
        there[0, page * 64:(page + 1) * 64] = False
    k[0, :, ~there[0]], v[0, :, ~there[0]] = 0.0, 0.0
    for causal in (False, True):
        compare(cache, k, v, queries(2, 2, 150, D, dtype), [m, m - 3], causal, dtype, there)


@pytest.mark.parametrize("D,dtype,m", [
    (128, "bf16", 120 * 64 - 5),                # 15 pieces
    (64, "f32", 120 * 64 - 60),
    (64, "bf16", 400 * 64 - 1),                 # 50 pieces
    (128, "f32", 300 * 64),                     # 38 pieces
])
def test_lists_in_many_pieces(D, dtype, m):
    cache, k, v = filled(1, 1, D, m, seed=3)
    compare(cache, k, v, queries(1, 1, 200, D, dtype), [m], True, dtype)


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "bf16"), (64, "f32")])
def test_pieces_of_more_pages_than_a_wave_fetches_at_once(D, dtype):
    """64 lists of two tiles each, in four pieces of some 150 pages, a run of them left out."""
    m = 150 * 4 * 64 - 7
    cache, k, v = filled(1, 2, D, m, seed=4)
    cache.table[0, 60:71] = -1
    cache.table[0, 128] = -1
    there = torch.ones(1, m, dtype=torch.bool)
    there[0, 60 * 64:71 * 64] = there[0, 128 * 64:129 * 64] = False
    k[0, :, ~there[0]], v[0, :, ~there[0]] = 0.0, 0.0
    many = vsa2.KVCache(cache.pool, cache.table.repeat(32, 1))
    q = queries(32, 2, 140, D, dtype)
    lengths = [m - 64 * b for b in range(32)]
    got = vsa2.attn_cache(many, q, i32(lengths))
    for b in (0, 1, 17, 31):
        check([x[b:b + 1] for x in got], plain(k, v, q[b:b + 1], [lengths[b]], False, there), dtype)
