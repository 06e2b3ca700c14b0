"""The cache's operators as they are used together: lists assigned, tokens written, copied and
attended, against a model that keeps every sequence's tokens in order."""
import math
import os
import sys

import pytest
import torch

import around_reference as ref
import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def read_back(x):
    """What the cache makes of rows [..., D], in 64 bits."""
    codes, e = ref.quantised(x)
    return ref.VALUES[codes] * torch.pow(2.0, e.double())[..., None]


class Model:
    """Keys and values [tokens, heads, D] of every sequence, in order."""

    def __init__(self, batch, heads, D):
        self.k = [torch.zeros(0, heads, D, dtype=torch.float64) for _ in range(batch)]
        self.v = [x.clone() for x in self.k]

    def assign(self, length, source, drop):
        for name in ("k", "v"):
            old, new = getattr(self, name), []
            for b, n in enumerate(length):
                src = b if source is None else source[b]
                first, num = (0, 0) if drop is None else drop[b]
                x = old[src] if src >= 0 else old[0][:0]
                new.append(torch.cat([x[:64 * first], x[64 * (first + num):]])[:n])
            setattr(self, name, new)

    def write(self, k, v, count):
        for b, n in enumerate(count):
            self.k[b] = torch.cat([self.k[b], read_back(k[b, :, :n].transpose(0, 1))])
            self.v[b] = torch.cat([self.v[b], read_back(v[b, :, :n].transpose(0, 1))])

    def attend(self, b, q, first=0, before=None):
        """Outputs [hq, n, D] of q over sequence b's tokens from `first` on, behind those of `before`."""
        k, v = self.k[b][first:], self.v[b][first:]
        if before is not None:
            k, v = torch.cat([before.k[0], k]), torch.cat([before.v[0], v])
        group = q.shape[0] // k.shape[1]
        out = torch.zeros(q.shape, dtype=torch.float64)
        for h in range(q.shape[0]):
            s = q[h].double() @ k[:, h // group].t() / math.sqrt(q.shape[-1])
            out[h] = torch.softmax(s, -1) @ v[:, h // group]
        return out


def near(got, want):
    """fp32 queries, the bound of test_gpu_attn_cache: (2 delta + 2^-19) W with sums of |q k| / 8 below 16
    (delta = 2^-16 + 2^-21) and W = sum p |v| below 3.5, in all below 2^-13."""
    assert ((got.double().cpu() - want).abs() <= 2.0 ** -13).all(), (got.double().cpu() - want).abs().max()


def test_serving_steps():
    """Samples of one prompt that fork, lose pages, write one token or many, end and start anew, in a
    pool that fits them barely; their tokens' order is the model's after every step."""
    batch, heads, hq, D, m = 4, 2, 4, 64, 8
    g = torch.Generator().manual_seed(11)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pool_pages = 30
    prefix = vsa2.KVCache.empty(torch.full((1, 3), -1, dtype=torch.int32, device="cuda"), pool_pages, heads, D)
    own = vsa2.KVCache(prefix.pool, torch.full((batch, m), -1, dtype=torch.int32, device="cuda"))
    refs = torch.zeros(pool_pages, dtype=torch.int32, device="cuda")
    clip, model = Model(1, heads, D), Model(batch, heads, D)
    k, v = (torch.randn(1, heads, 150, D, generator=g) for _ in range(2))
    assert vsa2.cache_assign(prefix, refs, ints(0), count=ints(150)).tolist() == [150]
    vsa2.cache_write(prefix, k.cuda(), v.cuda(), ints(0))
    clip.write(k, v, [150])
    # length kept of the source, source, (first, number) of the pages that leave, new tokens
    steps = [
        ([0, 0, 0, 0], None, None, [70, 1, 64, 65]),
        ([70, 1, 64, 65], None, None, [1, 1, 1, 1]),
        ([71, 71, 65, 65], [0, 0, 2, 2], None, [1, 1, 1, 0]),             # forks, last pages shared and copied
        ([72, 72, 66, 65], None, None, [30, 90, 1, 1]),
        ([102, 98, 100, 64], [0, 1, 1, 3], [(0, 0), (0, 1), (0, 0), (0, 0)], [60, 1, 1, 1]),     # one loses its first page
        ([50, 99, 0, 65], [0, 1, -1, 3], None, [1, 1, 40, 1]),            # cut back, ended and started anew
        ([51, 100, 40, 66], [1, 1, 2, 1], None, [1, 1, 1, 1]),
    ]
    for length, source, drop, count in steps:
        room = vsa2.cache_assign(own, refs, ints(*length), source=None if source is None else ints(*source),
                                 drop=None if drop is None else torch.tensor(drop, dtype=torch.int32, device="cuda"),
                                 count=ints(*count))
        assert room.tolist() == count
        n = max(max(count), 1)
        k, v = (torch.randn(batch, heads, n, D, generator=g) for _ in range(2))
        vsa2.cache_write(own, k.cuda(), v.cuda(), ints(*length), room)
        model.assign(length, source, drop)
        model.write(k, v, count)
        total = [a + b for a, b in zip(length, count)]
        assert [len(x) for x in model.k] == total
        # every page's count is how many entries name it
        entries = torch.cat([prefix.table.flatten(), own.table.flatten()])
        want = torch.bincount(entries[entries >= 0].long(), minlength=pool_pages)
        assert torch.equal(refs.long(), want)
        q = torch.randn(batch, hq, 2, D, generator=g)
        o, _ = vsa2.attn_cache_shared(prefix, own, q.cuda(), ints(150), ints(*total))
        w, _ = vsa2.attn_cache_scored(own, q.cuda(), ints(*total), window=33)
        for b in range(batch):
            near(o[b], model.attend(b, q[b], before=clip))
            for i in range(2):
                near(w[b, :, i:i + 1], model.attend(b, q[b, :, i:i + 1], first=max(0, total[b] - 2 + i - 32)))
    # compaction: every second token of two sequences, into lists of a second table
    other = vsa2.KVCache(own.pool, torch.full((batch, m), -1, dtype=torch.int32, device="cuda"))
    kept = [list(range(i % 2, len(x), 2)) if i < 2 else [] for i, x in enumerate(model.k)]
    n = max(map(len, kept))
    index = torch.tensor([x + [0] * (n - len(x)) for x in kept], dtype=torch.int32, device="cuda")
    sizes = ints(*map(len, kept))
    zeros = ints(0, 0, 0, 0)
    assert torch.equal(vsa2.cache_assign(other, refs, zeros, count=sizes), sizes)
    vsa2.cache_copy(own, other, index, zeros, sizes)
    vsa2.cache_assign(own, refs, zeros)                       # the old lists are freed
    entries = torch.cat([prefix.table.flatten(), other.table.flatten()])
    assert torch.equal(refs.long(), torch.bincount(entries[entries >= 0].long(), minlength=pool_pages))
    for b in range(2):
        model.k[b], model.v[b] = model.k[b][kept[b]], model.v[b][kept[b]]
    q = torch.randn(batch, hq, 1, D, generator=g)
    o, lse = vsa2.attn_cache(other, q.cuda(), sizes)
    for b in range(2):
        near(o[b], model.attend(b, q[b]))
    assert (o[2:] == 0).all() and torch.isneginf(lse[2:]).all()


def test_sampling_example_against_a_plain_cache():
    """examples/video_layer.py's samples: the bound is that of its streaming (test_gpu_example.py)."""
    from test_gpu_example import plain
    from video_layer import Layer
    grid, h, w, old, samples, window = (8, 6, 9), 6, 9, 3, 3, 2
    layer = Layer(heads_q=6, heads_kv=3)
    g = torch.Generator().manual_seed(5)
    n, width = h * w, layer.heads_q * 128
    clip = torch.randn(1, old * n, width, generator=g).bfloat16()
    chunks = [torch.randn(samples, n, width, generator=g).bfloat16() for _ in range(4)]
    picks = [[0, 1, 2], [1, 1, 0], [2, 0, 1], [0, 0, 0]]
    got = list(layer.sample(clip.cuda(), [x.cuda() for x in chunks], [torch.tensor(p, dtype=torch.int32).cuda() for p in picks],
                            grid, window))
    gains = [t.double().cpu() for t in (layer.q_gain, layer.k_gain)]
    quant = lambda x: read_back(x.transpose(0, 1))
    rows = lambda x, frame: plain(layer, torch.cat([torch.zeros(1, frame * n, width, dtype=torch.float64), x[None].double()], 1),
                                  layer.w_qkv.double().cpu(), gains, (frame + x.shape[0] // n, h, w))
    _, k, v = rows(clip[0], 0)
    before = (quant(k), quant(v))
    own = [(before[0][:0], before[1][:0]) for _ in range(samples)]
    kept = 0
    for i, (x, pick, y) in enumerate(zip(chunks, picks, got)):
        passed = max(0, kept - (window - 1) * n) // 64 * 64
        kept += n - passed
        own = [tuple(t[passed:] for t in own[p]) for p in pick]
        for b in range(samples):
            q, k, v = (t[:, (old + i) * n:] for t in rows(x[b], old + i))
            own[b] = (torch.cat([own[b][0], quant(k)]), torch.cat([own[b][1], quant(v)]))
            kk, vv = (torch.cat(t) for t in zip(before, own[b]))
            assert len(own[b][0]) == kept
            kk, vv = (t.transpose(0, 1).repeat_interleave(2, 0) for t in (kk, vv))
            want = (torch.softmax(q @ kk.transpose(1, 2) / math.sqrt(128), -1) @ vv).transpose(0, 1).flatten(1)
            far = (y[b].double().cpu() - want).norm() / want.norm()
            assert far <= 2.0 ** -4, (i, b, float(far))


def test_caches_of_another_gpu_are_refused():
    """As in test_gpu_other_device.py: the number that a cache was made on is planted."""
    table = torch.zeros(1, 1, dtype=torch.int32).cuda()
    cache, other = vsa2.KVCache.empty(table, 1, 1, 64), vsa2.KVCache.empty(table.clone(), 1, 1, 64)
    q, one = torch.randn(1, 1, 4, 64, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    refs, index = torch.ones(1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    before = other.pool.clone()
    cache.device += 1
    for call in (lambda: vsa2.cache_assign(cache, refs, one), lambda: vsa2.cache_copy(cache, other, index, one),
                 lambda: vsa2.cache_copy(other, cache, index, one), lambda: vsa2.attn_cache_shared(cache, other, q, one, one),
                 lambda: vsa2.attn_cache_shared(other, cache, q, one, one), lambda: vsa2.attn_cache_scored(cache, q, one)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert torch.equal(other.pool, before) and refs.item() == 1
    with pytest.raises(ValueError, match="refs: expected"):
        vsa2.cache_assign(other, refs.repeat(2), one)
    with pytest.raises(ValueError, match="slope: expected"):
        vsa2.attn_cache_scored(other, q, one, slope=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError, match="span: expected"):
        vsa2.attn_cache_scored(other, q, one, span=torch.zeros(1, 4, dtype=torch.int32, device="cuda"))
    with pytest.raises(vsa2.Vsa2Error, match="VSA2_ERR_VALUE"):
        vsa2.attn_cache_scored(other, q, one, cap=-2.0)
    lists = vsa2.KVCache(other.pool, table.view(1, 1, 1))
    with pytest.raises(ValueError, match="table: expected"):
        vsa2.cache_assign(lists, refs, one)
