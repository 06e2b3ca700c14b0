"""What no row sees reaches no bit of the attentions' results: equal calls on pools whose stale
bytes differ (behind a list's end, between two rows' ranges), or with other queries in the places
past a call's counts, give equal outputs.  NaN there is tested elsewhere; these are finite bytes
and queries of other requests."""
import pytest
import torch

import around_reference as ref
import paper_2609_32882_amd as vsa2
from test_gpu_attn_cache import gpu, make
from test_gpu_attn_cache_scored import options, run, seen

pytestmark = pytest.mark.gpu

# (code, power) of stale places: a fresh page's zeros, the largest finite code, sizes as real ones have
STALE = [(0x00, 0), (0x7e, 150), (0xb1, 118)]
SIZES = (0.0, 1.0, 2.0 ** 12, float("nan"))          # of queries past the counts


def filled(pool, table, D, unseen, code, power):
    """The pool with the places in unseen bool [batch, positions] holding this code and power."""
    pool = pool.clone()
    for b, pos in unseen.nonzero().tolist():
        for h in range(pool.shape[1]):
            page = ref.page_for(table, b, h, pos, pool.shape[0])
            if page is None:
                continue
            for x, at in enumerate(ref.offsets(pos % 64, D)):
                pool[page, h, at] = code if x < 2 else power
    return pool


def padded(q, counts, size):
    """Queries with those past the counts (None: none) multiplied by size."""
    q = q.clone()
    for b in range(q.shape[0]):
        if counts is not None:
            q[b, :, int(counts[b]):] *= size
    return q


def alike(a, b):
    for x, y in zip(a, b):
        bits = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
        assert torch.equal(x.view(bits), y.view(bits)), (x.float() - y.float()).abs().max()


# as in test_gpu_attn_cache_scored.py, then cap, slope, window, sink, span
SCORED = [
    ((3, 10, 2, 128, 1, 9, [1, 65, 570], None, False, False, "bf16"), 30.0, False, 0, 0, None),
    ((2, 6, 2, 64, 5, 5, [130, 300], [5, 3], True, False, "bf16"), 30.0, True, 17, 3, None),
    ((2, 4, 2, 64, 20, 6, [380, 333], [20, 7], False, False, "bf16"), 15.0, False, 0, 0, "holes"),
    ((2, 2, 1, 64, 130, 5, [310, 260], [130, 40], False, False, "bf16"), 30.0, False, 0, 0, None),
    ((2, 2, 1, 64, 130, 5, [250, 130], [130, 77], True, False, "bf16"), 30.0, True, 65, 1, None),
    ((1, 2, 1, 128, 150, 9, [560], [100], False, False, "bf16"), 300.0, True, 0, 5, "holes"),
    ((1, 1, 1, 128, 140, 12, [760], [130], True, False, "bf16"), 0.0, True, 150, 130, None),
    ((1, 2, 1, 64, 140, 6, [370], [90], False, False, "f32"), 30.0, True, 0, 0, "holes"),
]


@pytest.mark.parametrize("i", range(len(SCORED)))
def test_scored_stale_places(i):
    case, *rest = SCORED[i]
    opt = options(case, *rest)
    x = make(case)
    unseen = ~seen(case, opt).any(1)
    got = [run(case, filled(x[0], x[1], case[3], unseen, *s), x, opt) for s in STALE]
    alike(got[0], got[1])
    alike(got[0], got[2])


@pytest.mark.parametrize("i", [i for i, c in enumerate(SCORED) if c[0][7]])
def test_scored_padded_queries(i):
    case, *rest = SCORED[i]
    opt = options(case, *rest)
    x = make(case)
    got = [run(case, x[0], (*x[:2], padded(x[2], x[4], size), *x[3:]), opt) for size in SIZES]
    for other in got[1:]:
        alike(got[0], other)


def steep(case, seed=3):
    """Like make(): the tokens of a list's last page have value rows 2^20 times those before it, and every
    row scores them some 12 below, so that the scale of the weights moves there and rows are lifted."""
    batch, hq, hkv, D, n, max_pages, lengths, counts, causal, lists, dtype = case
    pool, table, q, length, count = make(case, seed)
    g = torch.Generator().manual_seed(seed)
    u = torch.randn(D, generator=g)
    u *= D ** 0.25 / u.norm()                                   # u.u / sqrt(D) = 1
    m = max(lengths)
    k = 0.2 * torch.randn(batch, hkv, m, D, generator=g)
    v = torch.randn(batch, hkv, m, D, generator=g)
    for b in range(batch):
        last = (lengths[b] - 1) // 64 * 64
        k[b, :, :last] += 2 * u
        k[b, :, last:] -= 10 * u
        v[b, :, :last] *= 2.0 ** -10
        v[b, :, last:] *= 2.0 ** 10
    ref.write_reference(pool, table, k, v, [0] * batch, lengths)
    q = (u + 0.2 * torch.randn(batch, n, hq, D, generator=g)).to(q.dtype).transpose(1, 2)
    return pool, table, q, length, count


PLAIN = [
    (2, 10, 2, 128, 1, 5, [65, 290], None, False, False, "bf16"),
    (2, 4, 2, 64, 20, 4, [150, 210], [20, 5], False, False, "bf16"),
    (1, 1, 1, 64, 140, 4, [150], None, False, False, "bf16"),
    (2, 2, 1, 128, 140, 6, [150, 280], [140, 100], False, False, "bf16"),
    (1, 2, 2, 128, 150, 4, [200], None, True, False, "bf16"),
    (1, 2, 1, 64, 140, 6, [330], [70], False, False, "f32"),
]




@pytest.mark.parametrize("i", [i for i, c in enumerate(PLAIN) if c[7]])
def test_padded_queries(i):
    case = PLAIN[i]
    pool, table, q, length, count = make(case)
    cache = vsa2.KVCache(pool.cuda(), table.cuda())
    prefix = vsa2.KVCache(cache.pool, table[:1].contiguous().cuda())          # the first list as the one that all share
    for call in (lambda y: vsa2.attn_cache(cache, y, length.cuda(), gpu(count), causal=case[8]),
                 lambda y: vsa2.attn_cache_shared(prefix, cache, y, length[:1].cuda(), length.cuda(), gpu(count), causal=case[8])):
        got = [call(padded(q, count, size).cuda()) for size in SIZES]
        for other in got[1:]:
            alike(got[0], other)


@pytest.mark.parametrize("i", range(len(PLAIN)))
@pytest.mark.parametrize("data", [make, steep])
def test_stale_places(i, data):
    case = PLAIN[i]
    pool, table, q, length, count = data(case)
    unseen = torch.arange(case[5] * 64) >= length[:, None]
    caches = [vsa2.KVCache(filled(pool, table, case[3], unseen, *s).cuda(), table.cuda()) for s in STALE]
    first = table[:1].contiguous().cuda()                    # the first list as the one that all share
    for call in (lambda c: vsa2.attn_cache(c, q.cuda(), length.cuda(), gpu(count), causal=case[8]),
                 lambda c: vsa2.attn_cache_shared(vsa2.KVCache(c.pool, first), c, q.cuda(), length[:1].cuda(), length.cuda(),
                                                  gpu(count), causal=case[8])):
        got = [call(c) for c in caches]
        alike(got[0], got[1])
        alike(got[0], got[2])
