"""Page lists assigned, and tokens copied between lists: exactly what the plain forms give."""
import random

import pytest
import torch

import around_reference as ref
import paging_reference as pref
import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu


def state(seed, batch, m, pages, heads=1, D=64, wild=False):
    """(pool, table, refs, generator): lists of any pages, refs as they hold them; wild: entries that
    name no page, and pages that other tables hold."""
    g = torch.Generator().manual_seed(seed)
    pool = torch.randint(0, 256, (pages, heads, 128 * D + 128), generator=g, dtype=torch.uint8)
    table = torch.randint(-1 if wild else 0, pages + (2 if wild else 0), (batch, m), generator=g, dtype=torch.int32)
    table = torch.where(torch.arange(m) < torch.randint(0, m + 1, (batch, 1), generator=g), table, -1).to(torch.int32)
    if wild:
        table[0, 0], table[-1, -1] = 2 ** 31 - 1, -2 ** 31
    named = table[(table >= 0) & (table < pages)].long()
    refs = torch.bincount(named, minlength=pages).to(torch.int32)
    if wild:
        refs += (torch.rand(pages, generator=g) < 0.2).int()
    return pool, table, refs, g


def run(pool, table, refs, length, room=None, **kw):
    cache = vsa2.KVCache(pool.cuda(), table.cuda())
    held = refs.cuda()
    got = vsa2.cache_assign(cache, held, length.cuda(), room=room, **{k: v if v is None else v.cuda() for k, v in kw.items()})
    return cache.pool.cpu(), cache.table.cpu(), held.cpu(), got.cpu()


def check(pool, table, refs, length, **kw):
    got = run(pool, table, refs, length, **kw)
    p, t, r = pool.clone(), table.clone(), refs.clone()
    room = pref.assign_reference(p, t, r, length, **kw)
    for name, a, b in zip(("table", "refs", "room", "pool"), (got[1], got[2], got[3], got[0]), (t, r, room, p)):
        assert torch.equal(a, b), name
    return got


@pytest.mark.parametrize("seed", range(40))
def test_assign_matches_the_plain_form(seed):
    """Any lists, lengths, sources, drops and counts; pools that run out of pages."""
    rnd = random.Random(seed)
    batch, m, pages = rnd.randint(1, 7), rnd.randint(1, 6), rnd.randint(2, 40)
    pool, table, refs, g = state(seed, batch, m, pages, heads=rnd.choice([1, 3]), D=rnd.choice([64, 128]), wild=rnd.random() < 0.5)
    length = torch.randint(-3, 64 * m + 10, (batch,), generator=g, dtype=torch.int32)
    if rnd.random() < 0.5:
        length = (length // 64 * 64 + rnd.choice([0, 1, 63])).to(torch.int32)
    source = torch.randint(-1, batch + 1, (batch,), generator=g, dtype=torch.int32) if rnd.random() < 0.7 else None
    drop = None
    if rnd.random() < 0.4:
        drop = torch.stack([torch.randint(-1, m + 1, (batch,), generator=g), torch.randint(-1, 3, (batch,), generator=g)],
                           1).to(torch.int32)
    count = torch.randint(-1, rnd.choice([2, 100, 300]), (batch,), generator=g, dtype=torch.int32) if rnd.random() < 0.9 else None
    check(pool, table, refs, length, source=source, drop=drop, count=count)


def test_assign_ends_of_32_bits():
    """Lengths, counts, sources and drops as far as 32 bits go."""
    pool, table, refs, _ = state(3, 5, 4, 40)
    top, low = 2 ** 31 - 1, -2 ** 31
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)
    check(pool, table, refs, ints(top, low, 65, 256, 100), count=ints(top, top, low, top, 1))
    check(pool, table, refs, ints(top, 10, 65, 256, 100), source=ints(top, low, 0, 4, 5), count=ints(1, top, 3, 0, 70),
          drop=ints(0, top, low, low, 2, 1, top, top, 1, 0).view(5, 2))


@pytest.mark.parametrize("batch", [1, 63, 1025, 5000])
def test_assign_many_sequences(batch):
    """More sequences than the planning workgroup has threads, and than it keeps numbers of in LDS;
    the last page of all is one that they share."""
    pages, m = 2 * batch + 9, 3
    pool = torch.randint(0, 256, (pages, 1, 8320), generator=torch.Generator().manual_seed(batch), dtype=torch.uint8)
    table = torch.full((batch, m), -1, dtype=torch.int32)
    table[:, 0] = 4
    table[batch // 2:, 0] = 7
    refs = torch.bincount(table[:, 0].long(), minlength=pages).to(torch.int32)
    length = torch.full((batch,), 20, dtype=torch.int32)
    count = (torch.arange(batch) % 4 * 40).to(torch.int32)
    check(pool, table, refs, length, count=count)
    refs[7] += 1                                    # held by another table, too
    check(pool, table, refs, length, count=count, source=(torch.arange(batch) // 2).to(torch.int32))


@pytest.mark.parametrize("pages", [16384, 16385, 65536, 65537, 70001, 150000])
def test_assign_large_pools(pages):
    """Free pages in later steps of the search; one workgroup, and one a step."""
    g = torch.Generator().manual_seed(pages)
    pool = torch.zeros(pages, 1, 8320, dtype=torch.uint8, device="cuda")
    refs = torch.ones(pages, dtype=torch.int32)
    free = torch.randperm(pages, generator=g)[:300].sort()[0]
    free = torch.cat([free, torch.tensor([pages - 1])]).unique()
    refs[free] = 0
    table = torch.full((6, 100), -1, dtype=torch.int32)
    taken = torch.where(refs == 1)[0][-6:]
    table[:, 0] = taken.to(torch.int32)
    refs[taken[0]] = 2                              # its copy comes first
    pool[taken[0]] = 9
    length = torch.full((6,), 10, dtype=torch.int32)
    for count in ([1] * 6, [640, 1, 6400, 64, 3000, 3]):
        cache, held = vsa2.KVCache(pool.clone(), table.cuda()), refs.cuda()
        room = vsa2.cache_assign(cache, held, length.cuda(), count=torch.tensor(count, dtype=torch.int32).cuda())
        small = torch.zeros(pages, 1, 1, dtype=torch.uint8)
        small[taken[0]] = 9
        t, r = table.clone(), refs.clone()
        want = pref.assign_reference(small, t, r, length, count=torch.tensor(count))
        assert torch.equal(cache.table.cpu(), t) and torch.equal(held.cpu(), r) and torch.equal(room.cpu(), want)
        assert torch.equal(cache.pool[:, 0].amin(1).cpu(), small[:, 0, 0]) and torch.equal(cache.pool[:, 0].amax(1).cpu(), small[:, 0, 0])


def test_assign_long_lists():
    """More entries than the planning workgroup trims, and than a launch has threads in one turn."""
    batch, m = 37, 30011
    pages = 3000
    table = torch.full((batch, m), -1, dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    table[:, ::31] = torch.randint(0, pages, table[:, ::31].shape, generator=g, dtype=torch.int32)
    refs = torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)
    pool = torch.zeros(pages, 1, 8320, dtype=torch.uint8)
    length = torch.randint(0, 64 * m, (batch,), generator=g, dtype=torch.int32) // 64 * 64
    check(pool, table, refs, length.to(torch.int32))
    check(pool, table, refs, length.to(torch.int32), source=torch.randint(0, batch, (batch,), generator=g, dtype=torch.int32))


def test_assign_rooms_streams_and_workspace():
    pool, table, refs, g = state(5, 4, 5, 30)
    length, count = torch.tensor([70, 0, 200, 130]).int(), torch.tensor([64, 100, 1, 0]).int()
    want = check(pool, table, refs, length, count=count)
    room = torch.full((4,), -7, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(pool, table, refs, length, count=count, room=room)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(room.cpu(), want[3])
    cache, held = vsa2.KVCache(pool.cuda(), table.cuda()), refs.cuda()
    st, need = vsa2.vsa2_cache_assign_workspace(cache.c)
    assert st == 0
    ws = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device="cuda")
    src = torch.tensor([3, 3, 2, -1], dtype=torch.int32).cuda()
    ln, ct = length.cuda(), count.cuda()
    st = vsa2.vsa2_cache_assign(cache.c, cache.table.data_ptr(), held.data_ptr(), ln.data_ptr(), src.data_ptr(), None,
                                ct.data_ptr(), None, ws.data_ptr() + 256, need, torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    p, t, r = pool.clone(), table.clone(), refs.clone()
    pref.assign_reference(p, t, r, length, source=src.cpu(), count=count)
    assert torch.equal(cache.table.cpu(), t) and torch.equal(held.cpu(), r) and torch.equal(cache.pool.cpu(), p)
    assert (ws[:256] == 0xa5).all() and (ws[256 + need:] == 0xa5).all()


def test_assign_replayed_in_a_graph():
    pool, _, _, g = state(6, 4, 6, 40)
    table, refs = torch.full((4, 6), -1, dtype=torch.int32), torch.zeros(40, dtype=torch.int32)
    cache, held = vsa2.KVCache(pool.cuda(), table.cuda()), refs.cuda()
    length, count = torch.zeros(4, dtype=torch.int32).cuda(), torch.full((4,), 70, dtype=torch.int32).cuda()
    source = torch.arange(4, dtype=torch.int32).cuda()
    step = lambda: vsa2.cache_assign(cache, held, length, source=source, count=count)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        room = step()
    t, r, p = cache.table.cpu(), held.cpu(), cache.pool.cpu()
    for ln, ct, src in (([70, 10, 0, 64], [1, 100, 5, 64], [0, 1, 2, 3]), ([71, 71, 30, 30], [1, 1, 1, 40], [0, 0, 1, 1]),
                        ([72, 72, 72, 72], [300, 1, 0, 1], [1, 1, 1, 1]), ([0, 0, 0, 9], [0, 0, 0, 0], [-1, -1, 0, 3])):
        for x, y in ((length, ln), (count, ct), (source, src)):
            x.copy_(torch.tensor(y, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = pref.assign_reference(p, t, r, length.cpu(), source=source.cpu(), count=count.cpu())
        assert torch.equal(cache.table.cpu(), t) and torch.equal(held.cpu(), r)
        assert torch.equal(room.cpu(), want) and torch.equal(cache.pool.cpu(), p)


# batch, heads, D, tokens of src, n, start, counts (None: n), which indices, lists per head of src / dst, two pools
COPIES = [
    (1, 1, 64, 64, 1, [0], None, "shift", False, False, False),
    (1, 2, 128, 200, 64, [0], None, "shift", False, False, True),
    (2, 1, 64, 300, 150, [5, 63], [150, 1], "shift", False, False, False),
    (3, 2, 128, 190, 130, [0, 64, 100], [0, 130, 77], "any", False, True, True),
    (2, 3, 64, 500, 257, [1, 40], None, "picked", True, False, False),
    (1, 1, 128, 700, 300, [60], None, "picked", False, False, True),
    (2, 2, 64, 200, 140, [-70, 150], None, "wild", False, False, False),
    (2, 1, 128, 256, 128, [0, 128], None, "same", False, False, True),
    (2, 1, 128, 256, 190, [3, 0], None, "back", False, False, True),
]


@pytest.mark.parametrize("case", COPIES, ids=["%dx%d-D%d-%d-n%d-%s" % (*c[:5], c[7]) for c in COPIES])
def test_copy_matches_the_plain_form(case):
    batch, heads, D, tokens, n, start, counts, kind, lists_a, lists_b, two = case
    g = torch.Generator().manual_seed(n)
    ma, mb = -(-tokens // 64), 5
    pages = batch * (ma + mb) + 3
    pool = torch.randint(0, 256, (pages, heads, 128 * D + 128), generator=g, dtype=torch.uint8)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    ta, tb = order[:batch * ma].view(batch, ma), order[batch * ma:batch * (ma + mb)].view(batch, mb)
    per_head = lambda t: torch.stack([t.flatten().roll(h).view(t.shape) for h in range(heads)], 1).contiguous()
    ta, tb = per_head(ta) if lists_a else ta.clone(), per_head(tb) if lists_b else tb.clone()
    at = torch.arange(n)
    index = {"shift": (at + tokens - n).expand(batch, n), "any": torch.randint(0, tokens, (batch, n), generator=g),
             "picked": torch.stack([torch.randperm(tokens, generator=g)[:n].sort()[0] for _ in range(batch)]),
             "wild": torch.randint(-40, tokens + 60, (batch, n), generator=g), "same": at.expand(batch, n),
             "back": (n - 1 - at).expand(batch, n)}[kind].to(torch.int32).contiguous()
    if kind == "wild":
        index[0, 3], index[1, 5] = 2 ** 31 - 1, -2 ** 31
        ta[0, 1], tb[1, 3] = -1, pages
    dst = torch.randint(0, 256, pool.shape, generator=g, dtype=torch.uint8) if two else pool
    start, count = torch.tensor(start, dtype=torch.int32), None if counts is None else torch.tensor(counts, dtype=torch.int32)
    want = pref.copy_reference(pool, ta, dst.clone(), tb, index, start, count)
    a = pool.cuda()
    b = dst.cuda() if two else a
    vsa2.cache_copy(vsa2.KVCache(a, ta.cuda()), vsa2.KVCache(b, tb.cuda()), index.cuda(), start.cuda(),
                    None if count is None else count.cuda())
    assert torch.equal(b.cpu(), want) and (not two or torch.equal(a.cpu(), pool))


def test_copied_tokens_read_alike():
    """A compacted list gives the attention the same tokens, whatever page they are on."""
    g = torch.Generator().manual_seed(2)
    table = torch.arange(20, dtype=torch.int32).view(2, 10).cuda()
    cache = vsa2.KVCache.empty(table[:, :6].contiguous(), 20, 2, 128)
    dst = vsa2.KVCache(cache.pool, table[:, 6:].contiguous())
    k = torch.randn(2, 2, 384, 128, generator=g).bfloat16().cuda()
    start = torch.zeros(2, dtype=torch.int32).cuda()
    vsa2.cache_write(cache, k, k.flip(2), start)
    index = torch.stack([torch.randperm(384, generator=g)[:200].sort()[0] for _ in range(2)]).to(torch.int32).cuda()
    vsa2.cache_copy(cache, dst, index, start)
    kk, vv = vsa2.cache_read(cache, 384, start)
    for x, y in zip((kk, vv), vsa2.cache_read(dst, 200, start)):
        assert torch.equal(y, torch.stack([x[b][:, index[b].long()] for b in range(2)]))
