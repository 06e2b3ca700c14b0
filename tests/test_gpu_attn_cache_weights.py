"""How exactly bf16 attention over the 8-bit cache weighs the values, against the
plain 64-bit form on the same codes.

A weight that keeps 11 significant bits is off by at most 2^-12 of itself, an
eighth of what rounding the result to bf16 costs (2^-9 at the same place of the
binade).  The two are independent, so the error's root mean square is at most
sqrt(1 + 1/64) = 1.008 of the rounding's alone where no weights cancel; a result
that is smaller than its terms has that many more of the weights' share.  1.05
leaves room for it.  Weights of 8 bits would give up to sqrt(2)."""
import math

import pytest
import torch

import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

# batch, hq, hkv, D, n, length of the first sequence (others shorter), causal
CASES = {
    "one token, one piece": (3, 8, 2, 128, 1, 500, False),
    "one token, pieces": (1, 3, 3, 64, 1, 6001, False),
    "one token, many sequences": (16, 40, 8, 128, 1, 2900, False),
    "a few tokens": (2, 6, 2, 128, 20, 3000, True),
    "pairs of tiles": (16, 8, 8, 64, 32, 2000, True),
    "128 rows, D 64": (1, 4, 2, 64, 300, 2500, True),
    "128 rows, D 128": (2, 2, 2, 128, 200, 4000, False),
}
KINDS = ("even", "spread", "peaked")


def filled(batch, hkv, D, lengths, kind, seed=0):
    """A cache of random tokens and what it holds: (cache, k, v [batch, heads, m, D] in 64 bits)."""
    g = torch.Generator().manual_seed(seed)
    m = max(lengths)
    pages = -(-m // 64)
    table = torch.randperm(batch * pages, generator=g).to(torch.int32).view(batch, pages).cuda()
    cache = vsa2.KVCache.empty(table, batch * pages, hkv, D)
    k, v = (torch.randn(batch, hkv, m, D, generator=g) for _ in range(2))
    if kind == "spread":        # values of very different sizes side by side
        v = v * 2.0 ** torch.randint(-12, 13, (batch, hkv, m, 1), generator=g)
    if kind == "peaked":
        k = 8 * k
    start = torch.zeros(batch, dtype=torch.int32).cuda()
    vsa2.cache_write(cache, k.cuda(), v.cuda(), start)
    k, v = vsa2.cache_read(cache, m, start, dtype=torch.float32)
    return cache, k.double(), v.double()


def plain(k, v, q, lengths, causal):
    """o [batch, heads, n, D] in 64 bits."""
    batch, hq, n, D = q.shape
    group = hq // k.shape[1]
    o = torch.zeros(batch, hq, n, D, dtype=torch.float64, device=q.device)
    for b in range(batch):
        limit = lengths[b] - torch.arange(n - 1, -1, -1, device=q.device) * int(causal)
        hidden = torch.arange(k.shape[2], device=q.device) >= limit[:, None]
        for h in range(hq):
            s = q[b, h].double() @ k[b, h // group].t() / math.sqrt(D)
            o[b, h] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ v[b, h // group]
    return o


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", CASES)
def test_weights_cost_little_beside_the_results_rounding(name, kind):
    batch, hq, hkv, D, n, longest, causal = CASES[name]
    lengths = [longest - 37 * b for b in range(batch)]
    cache, k, v = filled(batch, hkv, D, lengths, kind)
    q = torch.randn(batch, hq, n, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    length = torch.tensor(lengths, dtype=torch.int32).cuda()
    o, _ = vsa2.attn_cache(cache, q, length, causal=causal)
    want = plain(k, v, q, lengths, causal)
    least = (want.bfloat16().double() - want).square().mean().sqrt()
    far = (o.double() - want).square().mean().sqrt()
    assert far <= 1.05 * least, float(far / least)


@pytest.mark.parametrize("batch,n", [(512, 1), (256, 140)])
def test_many_small_weights_beside_a_large_one(batch, n):
    """20,000 tokens of 2^-23 of the largest weight each, alone in half of the elements: their
    sum there keeps the result's 8 bits.  In 16 bits, with the largest weight at 2^7, such a
    weight is a whole multiple of 2^-24 at 2^-16, so off by 2^-9 of itself at most; 2^-9 more is
    the result's rounding.  So many sequences (of the same pages) that no list is cut."""
    D, m = 128, 20001
    k = torch.zeros(1, 1, m, D)
    v = torch.zeros(1, 1, m, D)
    k[0, 0, 0, 0] = 16.0                        # the large weight's logit: 16 q_0 / sqrt(D)
    v[0, 0, 0, :64], v[0, 0, 1:, 64:] = 1.0, 1.0
    pages = -(-m // 64)
    table = torch.arange(pages, dtype=torch.int32).view(1, -1).cuda()
    cache = vsa2.KVCache.empty(table, pages, 1, D)
    vsa2.cache_write(cache, k.cuda(), v.cuda(), torch.zeros(1, dtype=torch.int32).cuda())
    cache = vsa2.KVCache(cache.pool, table.repeat(batch, 1))
    q = torch.zeros(batch, 1, n, D)
    q[..., 0] = 11.25
    o, _ = vsa2.attn_cache(cache, q.bfloat16().cuda(), torch.full((batch,), m, dtype=torch.int32).cuda())
    small = math.exp(-16 * 11.25 / math.sqrt(D))
    assert 2.0 ** -23 < small < 2.0 ** -22.5
    total = 1 + (m - 1) * small
    assert (o[..., 64:].double() - (m - 1) * small / total).abs().max() <= 2.0 ** -8 * (m - 1) * small / total
    assert (o[..., :64].double() - 1 / total).abs().max() <= 2.0 ** -9


def test_small_values_under_the_weight_beside_large_ones_without():
    """All weight on a token whose values are 2^-60 of its neighbours', which weigh nothing."""
    D = 64
    for n in (1, 140):
        for at in (5, 130):
            k = torch.full((1, 1, 200, D), -8.0)
            v = torch.full((1, 1, 200, D), 2.0 ** 30)
            k[0, 0, at], v[0, 0, at] = 8.0, 2.0 ** -30
            cache = vsa2.KVCache.empty(torch.arange(4, dtype=torch.int32).view(1, 4).cuda(), 4, 1, D)
            vsa2.cache_write(cache, k.cuda(), v.cuda(), torch.zeros(1, dtype=torch.int32).cuda())
            q = torch.full((1, 1, n, D), 8.0).bfloat16().cuda()       # logits of 512 and -512
            o, _ = vsa2.attn_cache(cache, q, torch.tensor([200], dtype=torch.int32).cuda())
            assert (o == 2.0 ** -30).all()


@pytest.mark.parametrize("n", [1, 20, 140])
def test_large_values_without_weight_after_small_ones_with_it(n):
    """The weight is on the first page, whose values are 2^-70 of the later pages'."""
    D, m = 64, 500
    k, v = torch.full((1, 2, m, D), -8.0), torch.full((1, 2, m, D), 2.0 ** 30)
    k[:, :, 3], v[:, :, :64] = 8.0, 2.0 ** -40
    cache = vsa2.KVCache.empty(torch.arange(8, dtype=torch.int32).view(1, 8).cuda(), 8, 2, D)
    vsa2.cache_write(cache, k.cuda(), v.cuda(), torch.zeros(1, dtype=torch.int32).cuda())
    q = torch.full((1, 4, n, D), 8.0).bfloat16().cuda()
    o, lse = vsa2.attn_cache(cache, q, torch.tensor([m], dtype=torch.int32).cuda(), causal=True)
    assert (o == 2.0 ** -40).all() and (lse == 512).all()
