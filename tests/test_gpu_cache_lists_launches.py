"""Page lists assigned by several launches: lists and pools beyond what one workgroup takes, with pages that
leave the lists and pools that run out, exactly as the plain form."""
import pytest
import torch

import paging_reference as pref
import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

PAGE_BYTES = 128 * 64 + 128

# batch, max_pages, pages of the pool, lists taken from others, pages left out.  One workgroup takes up to 1,024
# sequences with 6,144 entries (3,400 where they stay in their places) in a pool of 65,536 pages.
CASES = [
    (40, 700, 3000, False, False), (40, 700, 3000, False, True),                # trimmed; saved and written
    (40, 180, 1500, True, False), (40, 180, 1500, True, True),                  # by columns; saved and written
    (40, 60, 500, True, False), (40, 60, 500, True, True), (40, 60, 500, False, True),      # one workgroup
    (1100, 3, 1500, True, False), (1100, 3, 1500, True, True), (1100, 3, 1500, False, False),
    (2500, 2, 1300, True, False),                                               # too many for columns
    (30, 5, 65600, False, False), (30, 5, 65600, True, True), (1030, 3, 65600, True, False),
    (40, 60, 140000, True, False),
]
IDS = ["%dx%d-%d%s%s" % (*c[:3], "-source" * c[3], "-drop" * c[4]) for c in CASES]


def state(case, seed):
    """(table, refs, length, options): lists whose last pages are shared, by sequences that fork and by other
    tables; requests that some pools serve and others do not."""
    batch, m, pages, fork, leave = case
    g = torch.Generator().manual_seed(seed)
    rnd = lambda lo, hi, *shape: torch.randint(lo, hi, shape or (batch,), generator=g, dtype=torch.int32)
    used = min(pages - 20, batch * m // 3 + 5)
    named = torch.randperm(pages, generator=g)[:used].to(torch.int32)
    table = named[rnd(0, used, batch, m).long()]
    table = torch.where(torch.arange(m) < rnd(0, m + 1)[:, None], table, -1).to(torch.int32)
    table[rnd(0, batch, 3).long(), rnd(0, m, 3).long()] = torch.tensor([pages, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    refs = torch.bincount(table[(table >= 0) & (table < pages)].long(), minlength=pages).to(torch.int32)
    # all but some of the other pages are another table's, which holds a few of these lists' pages, too
    others = torch.ones(pages, dtype=torch.int32)
    others[named.long()] = (torch.rand(used, generator=g) < (1.0, 0.1, 0.1)[seed % 3]).int()     # all: nothing gets free
    others[torch.randperm(pages, generator=g)[:(3, 60, 400)[seed % 3]]] = 0
    refs += others
    length = rnd(-3, 64 * m + 10)
    length[rnd(0, batch, 1 + batch // 2).long()] = int(rnd(1, 64, 1))           # last pages that are not full
    kw = dict(source=None, drop=None)
    if fork:
        kw["source"] = torch.where(torch.rand(batch, generator=g) < 0.05, -1, rnd(0, 1 + batch // 4)).to(torch.int32)
    if leave:
        kw["drop"] = torch.stack([rnd(-1, m), rnd(-1, 1 + m // 2)], 1)
    count = rnd(0, 3)
    count[rnd(0, batch, 3).long()] = 64 * 9                                     # a few that take many pages
    return table, refs, length, dict(kw, count=count)


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_matches_the_plain_form(case, seed):
    table, refs, length, kw = state(case, seed)
    marks = (torch.arange(case[2]) % 251).to(torch.uint8)                       # every byte of a page
    pool = marks.cuda()[:, None, None].expand(-1, 1, PAGE_BYTES).contiguous()
    cache, held = vsa2.KVCache(pool, table.cuda()), refs.cuda()
    room = vsa2.cache_assign(cache, held, length.cuda(), **{k: v if v is None else v.cuda() for k, v in kw.items()})
    t, r, small = table.clone(), refs.clone(), marks[:, None, None].clone()
    want = pref.assign_reference(small, t, r, length, **kw)
    assert torch.equal(cache.table.cpu(), t) and torch.equal(held.cpu(), r) and torch.equal(room.cpu(), want)
    assert torch.equal(pool[:, 0].amin(1).cpu(), small[:, 0, 0]) and torch.equal(pool[:, 0].amax(1).cpu(), small[:, 0, 0])


@pytest.mark.parametrize("batch,m,pages", [(1100, 3, 1500), (200, 3, 65600), (900, 3, 2100), (900, 7, 2100)])
@pytest.mark.parametrize("free", [0, 1, 150])
def test_a_shared_last_page_that_all_holders_write(batch, m, pages, free):
    """Four pages, each the last one of a quarter of the sequences, two of them another table's, too: copies that
    are refused leave the page shared, and then its last holder, who needs none, has no room either."""
    table = torch.full((batch, m), -1, dtype=torch.int32)
    table[:, 0] = pages // 2
    table[:, 1] = torch.arange(batch) % 4 * 7 + 11
    refs = torch.ones(pages, dtype=torch.int32)
    refs[torch.randperm(pages, generator=torch.Generator().manual_seed(free))[:free]] = 0
    refs[pages // 2] = batch
    for i in range(4):
        refs[11 + 7 * i] = int((table[:, 1] == 11 + 7 * i).sum()) + (i >= 2)
    length = torch.full((batch,), 64 + 20, dtype=torch.int32)
    count = torch.ones(batch, dtype=torch.int32)
    count[::50] = 100
    marks = (torch.arange(pages) % 251).to(torch.uint8)
    for source in (None, torch.arange(batch, dtype=torch.int32).flip(0).contiguous()):
        pool = marks.cuda()[:, None, None].expand(-1, 1, PAGE_BYTES).contiguous()
        cache, held = vsa2.KVCache(pool, table.cuda()), refs.cuda()
        room = vsa2.cache_assign(cache, held, length.cuda(), source=None if source is None else source.cuda(), count=count.cuda())
        t, r, small = table.clone(), refs.clone(), marks[:, None, None].clone()
        want = pref.assign_reference(small, t, r, length, source=source, count=count)
        assert (want == 0).any() and (free == 0 or (want > 0).any())
        assert torch.equal(cache.table.cpu(), t) and torch.equal(held.cpu(), r) and torch.equal(room.cpu(), want)
        assert torch.equal(pool[:, 0].amin(1).cpu(), small[:, 0, 0]) and torch.equal(pool[:, 0].amax(1).cpu(), small[:, 0, 0])
