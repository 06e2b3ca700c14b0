"""The measured cases of the cache's page lists and of the attentions that read
shared and long lists.

What a server of a streaming model does around the paged 8-bit cache between two
calls of the model, and the attention calls it makes when several samples go on
from one clip, or when a clip is longer than what a token attends.  A case is one
call; its `kind` says which, its other fields are the sizes and types:

  assign   every sequence's page list becomes a part of another's (or its own),
           with room for new tokens: forks, windows, trims, frees
  copy     tokens picked by index from one cache's lists into another's, as they
           are stored
  shared   attention of new tokens over a list that several sequences share and
           then over each sequence's own
  scored   attention of new tokens over a list with capped scores, a bias by
           distance, a window behind some first tokens, and documents

Sizes are those of the workloads in `workload.py` (2 to 40 heads, D = 64 and 128),
whose frames are 1,792 (480p) and 3,840 (720p) tokens, and batches as a server has
them.

A page of 64 tokens of one KV head, 128*D + 128 bytes, as the plain forms read it:
  K codes  [4 t][D/64 u][4 g][16 r][16 b]  token 16 t + r, element 64 u + 16 g + b
  V codes  [D/16 c][4 g][16 r][4 t][4 i]   element 16 c + r, token 16 t + 4 g + i
  K exponents [16 r][4 t], V exponents [4 g][4 t][4 i], same tokens, plus 127
Codes are float8 e4m3; a value is code * 2^exponent.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64                   # tokens of a page
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
ZERO_POWER = 27             # the power byte of a row of zeros
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def _assign(batch, ctx, hkv, d=128, n=1, fork=1, drop=0, sink=0, ragged=False, **kw):
    """fork: sequences that go on from one; drop: pages that leave each list, after
    its first `sink` pages."""
    return dict(kind="assign", batch=batch, ctx=ctx, hkv=hkv, d=d, n=n, fork=fork, drop=drop, sink=sink, ragged=ragged, **kw)


def _copy(batch, ctx, n, hkv, d=128, picked=False, ragged=False, **kw):
    """picked: tokens from all over the list, in order; else the first tokens and the last ones."""
    return dict(kind="copy", batch=batch, ctx=ctx, n=n, hkv=hkv, d=d, picked=picked, ragged=ragged, **kw)


def _shared(groups, samples, n, prefix, ctx, hq, hkv, d=128, dtype="bf16", ragged=False, causal=False, **kw):
    return dict(kind="shared", groups=groups, samples=samples, batch=groups * samples, n=n, prefix=prefix, ctx=ctx,
                hq=hq, hkv=hkv, d=d, dtype=dtype, ragged=ragged, causal=causal, **kw)


def _scored(batch, n, ctx, hq, hkv, d=128, dtype="bf16", ragged=False, causal=False, cap=0.0, slope=False, window=0,
            sink=0, doc=0, **kw):
    """doc: tokens of a document, 0 for no documents."""
    return dict(kind="scored", batch=batch, n=n, ctx=ctx, hq=hq, hkv=hkv, d=d, dtype=dtype, ragged=ragged,
                causal=causal, cap=cap, slope=slope, window=window, sink=sink, doc=doc, **kw)


def listed():
    return [
        # serving, one new token of each of 64 sequences, one in 64 of which starts a page: latency
        _assign(64, 2048, 8, ragged=True, name="assign-token"),
        # 32 samples that go on from 8 of them, each with a last page of its own: copies of pages
        _assign(32, 17913, 8, fork=4, name="assign-fork"),
        # a window of 720p frames moves on: the oldest frame but the first leaves, room for a new one
        _assign(8, 38400, 8, d=64, n=3840, drop=60, sink=60, name="assign-frames"),
        # a few tokens of short lists, odd sizes: latency
        _copy(3, 1000, 37, 2, d=64, picked=True, ragged=True, name="copy-short"),
        # a 480p clip's first frame and its last tokens, which do not start at a page: bandwidth
        _copy(1, 35840, 29793, 12, name="copy-window"),
        # half the tokens of four clips, picked one by one
        _copy(4, 20000, 10007, 8, picked=True, name="copy-picked"),
        # one token of each of 32 samples of a 480p clip
        _shared(1, 32, 1, 35840, 2048, 40, 8, ragged=True, name="shared-token"),
        # a few tokens of five samples of each of two prompts, fp32
        _shared(2, 5, 3, 4001, 300, 12, 4, d=64, dtype="f32", ragged=True, causal=True, name="shared-few-f32"),
        # a 480p frame of two samples of a clip
        _shared(1, 2, 1792, 35840, 3584, 12, 12, name="shared-frame"),
        # one token of each of 16 sequences, capped scores
        _scored(16, 1, 38400, 40, 8, ragged=True, cap=30.0, name="scored-token"),
        # a few tokens each with all the options, fp32
        _scored(4, 17, 4001, 12, 4, d=64, dtype="f32", ragged=True, causal=True, cap=50.0, slope=True, window=1000,
                sink=4, doc=2300, name="scored-few-f32"),
        # a 480p frame over the first frame and the last five, biased by distance
        _scored(1, 1792, 35840, 12, 12, cap=30.0, slope=True, window=8960, sink=1792, name="scored-frame"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["assign", "copy", "shared", "shared", "scored", "scored"])
    d = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    hkv = rng.choice([1, 2, 4, 8, 12])
    group = rng.choice([1, 1, 2, 3, 5, 8])
    if kind == "assign":
        batch = _log(rng, 1, 200)
        ctx = _log(rng, 200, 300000 // batch + 200)
        fork = rng.choice([1, 1, 2, 3, 8])
        pages = ctx // PAGE
        drop = rng.randint(0, pages // 2) if rng.random() < 0.4 else 0
        sink = rng.randint(0, pages // 4)
        return _assign(batch, ctx, hkv, d=d, n=rng.choice([1, _log(rng, 1, ctx)]), fork=fork, drop=drop, sink=sink,
                       ragged=rng.random() < 0.6)
    if kind == "copy":
        batch = _log(rng, 1, 32)
        ctx = _log(rng, 64, 80000 // batch + 64)
        return _copy(batch, ctx, _log(rng, 1, ctx), hkv, d=d, picked=rng.random() < 0.5, ragged=batch > 1 and rng.random() < 0.6)
    if rng.random() < 0.7:
        n = rng.choice([1, 1, 1, _log(rng, 2, 32)])
        frames = False
    else:
        n, frames, hkv, group, dtype = _log(rng, 33, 1792), True, rng.choice([1, 2, 4]), min(group, 3), "bf16"
    if kind == "shared":
        groups, samples = (1, rng.choice([2, 3])) if frames else (rng.choice([1, 1, 2, 4]), _log(rng, 2, 32))
        prefix = _log(rng, 64, 35840)
        own_ctx = max(n, _log(rng, 64, 4096))
        return _shared(groups, samples, n, prefix, own_ctx, min(hkv, 8) * group, min(hkv, 8), d=d, dtype=dtype,
                       ragged=rng.random() < 0.6, causal=rng.random() < 0.5)
    batch = 1 if frames else _log(rng, 1, 32)
    ctx = _log(rng, 1792, 35840) if frames else max(n, _log(rng, 64, 600000 // batch))
    windowed = rng.random() < 0.5
    return _scored(batch, n, ctx, min(hkv, 8) * group, min(hkv, 8), d=d, dtype=dtype, ragged=batch > 1 and rng.random() < 0.6,
                   causal=rng.random() < 0.5, cap=rng.choice([0.0, 15.0, 30.0, 50.0]), slope=rng.random() < 0.5,
                   window=_log(rng, 1, ctx) if windowed else 0, sink=rng.choice([0, 1, 4, 100]) if windowed else 0,
                   doc=_log(rng, 64, ctx) if ctx > 64 and rng.random() < 0.4 else 0)


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------
def _pages(tokens):
    return -(-tokens // PAGE)


def _lengths(c, ctx=None):
    """Tokens that each sequence has in its list, uneven in a ragged batch."""
    ctx = c["ctx"] if ctx is None else ctx
    if not c["ragged"]:
        return [ctx] * c["batch"]
    return [max(1, ctx - (b * ctx * 3) // (4 * c["batch"]) - 13 * b) for b in range(c["batch"])]


def _counts(c):
    """Tokens of the call that each sequence has."""
    return [max(1, c["n"] - b % 3) if c["ragged"] else c["n"] for b in range(c["batch"])]


def _prefixes(c):
    """Tokens of each shared list."""
    return [max(1, c["prefix"] - 101 * g) if c["ragged"] else c["prefix"] for g in range(c["groups"])]


def _kept(c):
    """Of an assign: (source, tokens kept, (first page, pages) that leave) of every sequence."""
    out = []
    lens = _lengths(c)
    for b in range(c["batch"]):
        src = b - b % c["fork"]
        first = min(c["sink"], _pages(lens[src]))
        num = max(0, min(c["drop"], _pages(lens[src]) - first - 1))
        out.append((src, lens[src] - PAGE * num, (first, num)))
    return out


def _max_pages(c):
    return _pages(c["ctx"] + c["n"])


def _views(c, b):
    """(own position, limit, from, to) of each of sequence b's tokens in a scored call."""
    count, length = _counts(c)[b], _lengths(c)[b]
    out = []
    for i in range(count):
        p = length - count + i
        limit = max(0, p + 1 if c["causal"] else length)
        lo, hi = 0, length
        if c["doc"]:
            lo = max(p, 0) // c["doc"] * c["doc"]
            hi = lo + c["doc"]
        if c["window"]:
            lo = max(lo, p + 1 - c["window"])
        out.append((p, limit, lo, min(hi, limit)))
    return out


def work(c):
    d = c["d"]
    token = 2 * (d + 1)             # of one KV head in the cache
    if c["kind"] == "assign":
        copies = entries = 0
        lens = _lengths(c)
        for b, (src, kept, _) in enumerate(_kept(c)):
            moved = src != b or c["drop"] > 0
            entries += _pages(kept) if moved else 0
            entries += _pages(kept + c["n"]) - _pages(kept)
            copies += 1 if kept % PAGE and c["fork"] > 1 and (b % c["fork"] < c["fork"] - 1 and b + 1 < c["batch"]) else 0
            entries += _pages(lens[b]) if moved else 0
        return {"bytes": copies * 2 * c["hkv"] * PAGE * token + 16 * entries + 20 * c["batch"], "flops": 2 * entries}
    if c["kind"] == "copy":
        rows = sum(_counts(c))
        return {"bytes": rows * (2 * c["hkv"] * token + 4), "flops": rows * c["hkv"]}
    e = 4 if c["dtype"] == "f32" else 2
    rows = c["batch"] * c["n"] * c["hq"]
    ends = rows * (2 * d * e + 4)
    if c["kind"] == "shared":
        pairs = 0
        for b in range(c["batch"]):
            count, length = _counts(c)[b], _lengths(c)[b]
            before = _prefixes(c)[b // c["samples"]]
            pairs += sum(before + (max(0, length - (count - 1 - i)) if c["causal"] else length) for i in range(count))
        tokens = sum(_prefixes(c)) + sum(_lengths(c))
        return {"bytes": ends + tokens * c["hkv"] * token, "flops": 4.0 * d * pairs * c["hq"]}
    pairs = tokens = 0
    for b in range(c["batch"]):
        views = _views(c, b)
        sinks = min(c["sink"], max(v[1] for v in views))
        lo, hi = max(sinks, min(v[2] for v in views)), max(v[3] for v in views)
        tokens += sinks + max(0, hi - lo)
        pairs += sum(min(c["sink"], v[1]) + max(0, v[3] - max(v[2], min(c["sink"], v[1]))) for v in views)
    return {"bytes": ends + tokens * c["hkv"] * token, "flops": 4.0 * d * pairs * c["hq"]}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    _prepare[c["kind"]](c, gen, s)
    return s


def _pool(c, gen, pages):
    """Pages of values of about unit size."""
    d, hkv = c["d"], c["hkv"]
    pool = torch.empty(pages, hkv, 128 * d + 128, dtype=torch.uint8, device="cuda")
    for lo in range(0, pages, 4096):        # a page's values are alike: drawn in the order they are stored
        piece = pool[lo:lo + 4096]
        x = torch.randn(piece.shape[0], hkv, 128 * d, generator=gen, device="cuda") * 96
        piece[..., :128 * d] = x.clamp_(-E4M3_MAX, E4M3_MAX).to(E4M3).view(torch.uint8)
        piece[..., 128 * d:] = torch.randint(127 - 8, 127 - 5, (piece.shape[0], hkv, 128), generator=gen, device="cuda",
                                             dtype=torch.uint8)
    return pool


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _order(gen, pages):
    return torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)


def _queries(c, gen):
    q = 1.5 * torch.randn(c["batch"], c["n"], c["hq"], c["d"], generator=gen, device="cuda")
    return q.to(DTYPES[c["dtype"]])


def _prepare_assign(c, gen, s):
    """A pool whose pages the lists hold in no order, with a spare one behind it
    that the plain form copies onto itself; how often each page is held."""
    lens, m, b = _lengths(c), _max_pages(c), c["batch"]
    held = torch.tensor([_pages(n) for n in lens], device="cuda")
    need = b * (_pages(c["n"]) + 2)
    pages = sum(_pages(n) for n in lens) + need
    s["store"] = torch.randint(0, 256, (pages + 1, c["hkv"], 128 * c["d"] + 128), generator=gen, device="cuda",
                               dtype=torch.uint8)
    s["pool"] = s["store"][:pages]
    order = _order(gen, pages)
    at = (held.cumsum(0) - held)[:, None] + torch.arange(m, device="cuda")
    mine = torch.arange(m, device="cuda") < held[:, None]
    s["table"] = torch.where(mine, order[torch.where(mine, at, 0)], -1).contiguous()
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device="cuda")
    s["refs"][order[:sum(_pages(n) for n in lens)].long()] = 1
    kept = _kept(c)
    s["source"] = _ints([k[0] for k in kept]) if c["fork"] > 1 else None
    s["length"] = _ints([k[1] for k in kept])
    s["drop"] = _ints([k[2] for k in kept]) if c["drop"] else None
    s["count"] = _ints(_counts(c))


def _prepare_copy(c, gen, s):
    """Two sets of lists over one pool, the tokens' indices."""
    lens, b = _lengths(c), c["batch"]
    m, mine = _pages(c["ctx"]), _pages(c["n"] + PAGE)
    total = b * (m + mine) + 3
    s["pool"] = _pool(c, gen, total)
    order = _order(gen, total)
    s["table"], s["to"] = order[:b * m].view(b, m), order[b * m:b * (m + mine)].view(b, mine)
    s["count"] = _ints(_counts(c)) if c["ragged"] else None
    s["start"] = torch.randint(0, PAGE, (b,), generator=gen, device="cuda", dtype=torch.int32) if c["ragged"] else _ints([0] * b)
    index = torch.zeros(b, c["n"], dtype=torch.int32, device="cuda")
    for x, n in enumerate(lens):
        k = min(c["n"], n)
        if c["picked"]:
            index[x, :k] = torch.randperm(n, generator=gen, device="cuda")[:k].sort()[0]
        else:
            at = torch.arange(k, device="cuda")
            index[x, :k] = torch.where(at < k // 16, at, n - k + at)
    s["index"] = index


def _prepare_shared(c, gen, s):
    pre, mine = _pages(c["prefix"]), _pages(c["ctx"])
    total = c["groups"] * pre + c["batch"] * mine + 3
    s["pool"] = _pool(c, gen, total)
    order = _order(gen, total)
    s["shared"] = order[:c["groups"] * pre].view(c["groups"], pre)
    s["table"] = order[c["groups"] * pre:c["groups"] * pre + c["batch"] * mine].view(c["batch"], mine)
    s["prefix_length"], s["length"] = _ints(_prefixes(c)), _ints(_lengths(c))
    s["count"] = _ints(_counts(c)) if c["ragged"] else None
    s["q"] = _queries(c, gen)


def _prepare_scored(c, gen, s):
    m, b = _pages(c["ctx"]), c["batch"]
    s["pool"] = _pool(c, gen, b * m + 3)
    s["table"] = _order(gen, b * m + 3)[:b * m].view(b, m)
    lens, counts = _lengths(c), _counts(c)
    s["length"] = _ints(lens)
    s["count"] = _ints(counts) if c["ragged"] else None
    s["q"] = _queries(c, gen)
    s["slope"] = torch.rand(c["hq"], generator=gen, device="cuda") * (4.0 / c["ctx"]) if c["slope"] else None
    s["span"] = None
    if c["doc"]:
        at = s["length"][:, None] - _ints(counts)[:, None] + torch.arange(c["n"], device="cuda", dtype=torch.int32)
        lo = at.clamp_min(0) // c["doc"] * c["doc"]
        s["span"] = torch.stack([lo, lo + c["doc"]], -1).to(torch.int32).contiguous()


_prepare = {"assign": _prepare_assign, "copy": _prepare_copy, "shared": _prepare_shared, "scored": _prepare_scored}


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _heads_first(x):
    """[batch, tokens, heads, D] seen as [batch, heads, tokens, D]."""
    return x.transpose(1, 2)


# the framework's calls ----------------------------------------------------
def _own_assign(s):
    import paper_2609_32882_amd as vsa2
    cache = vsa2.KVCache(s["pool"], s["table"])
    room = vsa2.cache_assign(cache, s["refs"], s["length"], source=s["source"], drop=s["drop"], count=s["count"])
    return s["table"], s["refs"], room, s["pool"]


def _own_copy(s):
    import paper_2609_32882_amd as vsa2
    vsa2.cache_copy(vsa2.KVCache(s["pool"], s["table"]), vsa2.KVCache(s["pool"], s["to"]), s["index"], s["start"],
                    s["count"])
    return s["pool"]


def _own_shared(s):
    import paper_2609_32882_amd as vsa2
    return vsa2.attn_cache_shared(vsa2.KVCache(s["pool"], s["shared"]), vsa2.KVCache(s["pool"], s["table"]),
                                  _heads_first(s["q"]), s["prefix_length"], s["length"], s["count"],
                                  causal=s["case"]["causal"])


def _own_scored(s):
    import paper_2609_32882_amd as vsa2
    c = s["case"]
    return vsa2.attn_cache_scored(vsa2.KVCache(s["pool"], s["table"]), _heads_first(s["q"]), s["length"], s["count"],
                                  causal=c["causal"], cap=c["cap"], slope=s["slope"], window=c["window"],
                                  sink=c["sink"], span=s["span"])


_own = {"assign": _own_assign, "copy": _own_copy, "shared": _own_shared, "scored": _own_scored}


# the plain forms ----------------------------------------------------------
def _plain_assign(s):
    c, table, refs = s["case"], s["table"].long(), s["refs"]
    b, m = table.shape
    pages = refs.shape[0]
    seq, slot = torch.arange(b, device="cuda"), torch.arange(m, device="cuda")
    src = seq if s["source"] is None else s["source"].long()
    real = (src >= 0) & (src < b)
    length = torch.where(real, s["length"].long().clamp(0, PAGE * m), 0)
    count = s["count"].long().clamp_min(0)
    kept, wanted = (length + PAGE - 1) // PAGE, ((length + count + PAGE - 1) // PAGE).clamp_max(m)
    # the lists that the kept pages make, and how often every page is held then
    first, num = (torch.zeros_like(length),) * 2 if s["drop"] is None else s["drop"].long().unbind(1)
    at = slot + torch.where(slot >= first[:, None], num.clamp_min(0)[:, None], 0)
    shown = (slot < kept[:, None]) & (at < m)
    new = torch.where(shown, table[src.clamp(0, b - 1)[:, None], at.clamp_max(m - 1)], -1)
    named = (new >= 0) & (new < pages)
    new = torch.where(named, new, -1)
    for lists, one in ((table, -1), (new, 1)):
        fine = (lists >= 0) & (lists < pages)
        refs.index_add_(0, torch.where(fine, lists, 0).flatten(), (fine.to(torch.int32) * one).flatten())
    # last pages that a sequence writes into: a copy if another holds it, too; of
    # sequences that all write, the last keeps it
    last = new.gather(1, (kept - 1).clamp_min(0)[:, None])[:, 0]
    inside = (count > 0) & (length % PAGE != 0)
    writes = inside & (last >= 0)
    page = torch.where(writes, last, pages)
    writers = torch.zeros(pages + 1, dtype=torch.int32, device="cuda").index_add_(0, page, writes.to(torch.int32))
    final = torch.full((pages + 1,), -1, device="cuda").scatter_reduce_(0, page, seq, "amax")
    holds = torch.cat([refs, refs.new_zeros(1)])[page]
    copies = writes & (holds > 1) & ~((holds == writers[page]) & (final[page] == seq))
    # requests in order, free pages in order
    request = torch.cat([copies[:, None], (slot >= kept[:, None]) & (slot < wanted[:, None])], 1)
    rank = request.flatten().cumsum(0).view(b, m + 1) - 1
    free = refs == 0
    there = torch.where(free, free.cumsum(0) - 1, pages)
    ids = torch.full((pages + 1,), -1, device="cuda").scatter_(0, there, torch.arange(pages, device="cuda"))
    ids[pages] = -1
    given = torch.where(request, ids[rank.clamp(0, pages)], -1)
    fine = given >= 0
    refs.index_add_(0, given.clamp_min(0).flatten(), fine.flatten().to(torch.int32))
    copied = fine[:, 0]
    refs.index_add_(0, torch.where(copied, page, 0), -copied.to(torch.int32))
    s["store"][torch.where(copied, given[:, 0], pages)] = s["store"][torch.where(copied, page, pages)]
    new = torch.where(request[:, 1:], given[:, 1:], new)
    new = torch.where(copied[:, None] & (slot == kept[:, None] - 1), given[:, :1], new)
    s["table"].copy_(new)
    # tokens that have a place
    short = request[:, 1:] & (given[:, 1:] < 0)
    end = torch.where(short, slot, m).amin(1) * PAGE
    room = torch.minimum(count, end - length).clamp_min(0)
    own_page = ~inside | (writes & (copied | (torch.cat([refs, refs.new_zeros(1)])[page] == 1)))
    room = torch.where(own_page, room, 0)
    return s["table"], refs, room.to(torch.int32), s["pool"]


def _places(d, j):
    """Byte of every element of in-page tokens j [...]: K codes [..., D], V codes
    [..., D], and the two exponents [...], each within a page."""
    e = torch.arange(d, device=j.device)
    t, r, g, i = j // 16, j % 16, j // 4 % 4, j % 4
    k = ((t[..., None] * (d // 64) + e // 64) * 64 + e % 64 // 16 * 16 + r[..., None]) * 16 + e % 16
    v = 64 * d + ((e // 16) * 64 + g[..., None] * 16 + e % 16) * 16 + (t * 4 + i)[..., None]
    return k, v, 128 * d + r * 4 + t, 128 * d + 64 + g * 16 + t * 4 + i


def _plain_copy(s):
    c, pool = s["case"], s["pool"]
    heads = torch.arange(c["hkv"], device="cuda")[None, :, None, None]
    count = torch.full_like(s["start"], c["n"]) if s["count"] is None else s["count"]
    i = torch.arange(c["n"], device="cuda")
    live = i < count[:, None]
    at = torch.where(live, s["index"].long(), 0)
    to = torch.where(live, s["start"].long()[:, None] + i, s["start"].long()[:, None])     # the first token again
    at = torch.where(live, at, s["index"].long()[:, :1])
    from_page, to_page = (t.long().gather(1, x // PAGE)[:, None, :, None] for t, x in ((s["table"], at), (s["to"], to)))
    for a, b in zip(_places(c["d"], at % PAGE), _places(c["d"], to % PAGE)):
        a, b = (x[:, None] if x.dim() == 3 else x[:, None, :, None] for x in (a, b))
        pool[to_page, heads, b] = pool[from_page, heads, a]
    return pool


def _power(e):
    """2^e in fp32 of whole numbers -126 .. 127, by its bits: exact."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _unpacked(pool, table, d):
    """K and V [batch, Hkv, tokens, D] in fp32 of lists [batch, P]."""
    pages = pool[table.long()].transpose(1, 2)
    codes, exps = pages[..., :128 * d].view(E4M3), _power(pages[..., 128 * d:].int() - 127)
    k = codes[..., :64 * d].unflatten(-1, (4, d // 64, 4, 16, 16)).permute(0, 1, 2, 3, 6, 4, 5, 7)
    v = codes[..., 64 * d:].unflatten(-1, (d // 16, 4, 16, 4, 4)).permute(0, 1, 2, 6, 4, 7, 3, 5)
    ke = exps[..., :64].unflatten(-1, (16, 4)).transpose(-1, -2)
    ve = exps[..., 64:].unflatten(-1, (4, 4, 4)).transpose(-2, -3)
    b, h = pages.shape[:2]
    k = k.float().reshape(b, h, -1, d) * ke.reshape(b, h, -1, 1)
    v = v.float().reshape(b, h, -1, d) * ve.reshape(b, h, -1, 1)
    return k, v


def _seen(s, n, causal):
    """Which of the call's tokens are real, and their limits, [batch, n] each."""
    count = torch.full_like(s["length"], n) if s["count"] is None else s["count"]
    i = torch.arange(n, device="cuda")
    limit = s["length"][:, None].expand(-1, n)
    if causal:
        limit = limit - (count[:, None] - 1 - i)
    return i < count[:, None], limit, s["length"][:, None] - count[:, None] + i


def _softmax(scores):
    """Weights (not divided) and their sums and maxima of masked scores, in place."""
    top = scores.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p, total, (top + total.log())[..., 0]


def _plain_shared(s):
    c = s["case"]
    b, n, hq, hkv, d, g = c["batch"], c["n"], c["hq"], c["hkv"], c["d"], c["groups"]
    group, per = hq // hkv, c["samples"]
    kp, vp = _unpacked(s["pool"], s["shared"], d)
    k, v = _unpacked(s["pool"], s["table"], d)
    q = _heads_first(s["q"]).float().reshape(b, hkv, group * n, d)
    together = q.reshape(g, per, hkv, group * n, d).transpose(1, 2).reshape(g, hkv, per * group * n, d)
    far = torch.matmul(together, kp.transpose(-1, -2)).reshape(g, hkv, per, group * n, -1).transpose(1, 2)
    scores = torch.cat([far.reshape(b, hkv, group * n, -1), torch.matmul(q, k.transpose(-1, -2))], -1)
    del far
    scores = scores.mul_(1 / math.sqrt(d)).reshape(b, hkv, group, n, -1)
    real, limit, _ = _seen(s, n, c["causal"])
    before = s["prefix_length"].repeat_interleave(per)
    hidden = torch.cat([(torch.arange(kp.shape[2], device="cuda") >= before[:, None])[:, None].expand(b, n, -1),
                        torch.arange(k.shape[2], device="cuda") >= limit[..., None]], -1) | ~real[..., None]
    p, total, lse = _softmax(scores.masked_fill_(hidden[:, None, None], -math.inf))
    p = p.reshape(b, hkv, group * n, -1)
    far, near = p[..., :kp.shape[2]], p[..., kp.shape[2]:]
    far = far.reshape(g, per, hkv, group * n, -1).transpose(1, 2).reshape(g, hkv, per * group * n, -1)
    o = torch.matmul(far, vp).reshape(g, hkv, per, group * n, d).transpose(1, 2).reshape(b, hkv, group * n, d)
    o = (o + torch.matmul(near, v)) / total.clamp_min(1e-30).reshape(b, hkv, -1, 1)
    return o.reshape(b, hq, n, d).to(s["q"].dtype), lse.reshape(b, hq, n)


def _plain_scored(s):
    c = s["case"]
    b, n, hq, hkv, d = c["batch"], c["n"], c["hq"], c["hkv"], c["d"]
    group = hq // hkv
    k, v = _unpacked(s["pool"], s["table"], d)
    q = _heads_first(s["q"]).float().reshape(b, hkv, group * n, d)
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(1 / math.sqrt(d)).reshape(b, hkv, group, n, -1)
    if c["cap"]:
        scores = scores.div_(c["cap"]).tanh_().mul_(c["cap"])
    real, limit, place = _seen(s, n, c["causal"])
    j = torch.arange(k.shape[2], device="cuda")
    if s["slope"] is not None:
        away = (place[..., None] - j).abs().float()
        for h in range(hq):
            scores[:, h // group, h % group] -= s["slope"][h] * away
    inside = torch.ones(1, dtype=torch.bool, device="cuda")
    if c["window"]:
        inside = j > place[..., None] - c["window"]
    if s["span"] is not None:
        inside = inside & (j >= s["span"][..., :1]) & (j < s["span"][..., 1:])
    seen = (inside | (j < c["sink"])) & (j < limit[..., None]) & real[..., None]
    p, total, lse = _softmax(scores.masked_fill_(~seen[:, None, None], -math.inf))
    o = torch.matmul(p.reshape(b, hkv, group * n, -1), v) / total.clamp_min(1e-30).reshape(b, hkv, -1, 1)
    return o.reshape(b, hq, n, d).to(s["q"].dtype), lse.reshape(b, hq, n)


_plain = {"assign": _plain_assign, "copy": _plain_copy, "shared": _plain_shared, "scored": _plain_scored}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------
def exact(c, seed):
    if c["kind"] in ("assign", "copy"):
        return None                 # nothing is computed: the outputs are whole numbers and copies
    s = prepare(c, seed)
    return _exact[c["kind"]](s)


def _exact_list(pool, pages, h, d):
    """K and V [tokens, D] in 64 bits of KV head h of a list's pages."""
    at = _places(d, torch.arange(PAGE, device="cuda"))
    rows = pool[pages.long(), h]
    out = []
    for codes in range(2):
        two = torch.tensor(2.0, dtype=torch.float64, device="cuda").pow(rows[:, at[codes + 2]].double() - 127)
        out.append((rows[:, at[codes]].view(E4M3).double() * two[..., None]).flatten(0, 1))
    return out


def _exact_rows(s, of, score=None):
    """(o, lse) with the keys, values and visible places [n, tokens] that of(b, h) gives."""
    c = s["case"]
    b, n, hq, hkv, d = c["batch"], c["n"], c["hq"], c["hkv"], c["d"]
    group = hq // hkv
    o = torch.zeros(b, hq, n, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, hq, n), -math.inf, dtype=torch.float64, device="cuda")
    for x in range(b):
        count = _counts(c)[x]
        for h in range(hkv):
            k, v, shown = of(x, h)
            some = shown.any(-1)
            for y in range(h * group, (h + 1) * group):
                a = s["q"][x, :count, y].double() @ k.t() / math.sqrt(d)
                a = a if score is None else score(x, y, a)
                a = torch.where(shown, a, -math.inf)
                lse[x, y, :count] = torch.logsumexp(a, -1)
                o[x, y, :count][some] = torch.softmax(a[some], -1) @ v
    return o, lse


def _exact_shared(s):
    c = s["case"]
    before = {}

    def of(b, h):
        g = b // c["samples"]
        if (g, h) not in before:
            n = _prefixes(c)[g]
            before[g, h] = [x[:n] for x in _exact_list(s["pool"], s["shared"][g][:_pages(n)], h, c["d"])]
        kp, vp = before[g, h]
        length, count = _lengths(c)[b], _counts(c)[b]
        k, v = (x[:length] for x in _exact_list(s["pool"], s["table"][b][:_pages(length)], h, c["d"]))
        shown = torch.ones(count, kp.shape[0] + length, dtype=torch.bool, device="cuda")
        if c["causal"]:
            own_place = torch.arange(length, device="cuda")
            last = length - count + torch.arange(count, device="cuda")
            shown[:, kp.shape[0]:] = own_place <= last[:, None]
        return torch.cat([kp, k]), torch.cat([vp, v]), shown

    return _exact_rows(s, of)


def _exact_scored(s):
    c = s["case"]

    def of(b, h):
        length = _lengths(c)[b]
        k, v = (x[:length] for x in _exact_list(s["pool"], s["table"][b][:_pages(length)], h, c["d"]))
        shown = np.zeros((_counts(c)[b], length), dtype=bool)
        for i, (_, limit, lo, hi) in enumerate(_views(c, b)):
            shown[i, :min(c["sink"], limit)] = True
            shown[i, max(lo, 0):max(hi, 0)] = True
        return k, v, torch.from_numpy(shown).cuda()

    def score(b, y, a):
        if c["cap"]:
            a = c["cap"] * torch.tanh(a / c["cap"])
        if c["slope"]:
            at = torch.tensor([v[0] for v in _views(c, b)], dtype=torch.float64, device="cuda")
            a = a - s["slope"][y].double() * (at[:, None] - torch.arange(a.shape[1], device="cuda")).abs()
        return a

    return _exact_rows(s, of, score)


_exact = {"shared": _exact_shared, "scored": _exact_scored}
