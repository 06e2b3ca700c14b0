"""What the operators on page lists and the attentions over shared and scored lists refuse, on
the host: every call here fails (or has nothing to do) before any device work, so no pointer
is followed."""
import ctypes

import pytest

vsa2 = pytest.importorskip("paper_2609_32882_amd")

FAKE, MISALIGNED = 0x10000, 0x10008
BIG = 1 << 40
NAME = vsa2.STATUS_NAMES


def rows(ptr=FAKE, b=1 << 20, h=128, t=1024):
    return vsa2.vsa2_rows(ptr, b, h, t)


def cache(**kw):
    c = vsa2.vsa2_cache(4, 4, 128, 10, 6, 1, FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def scores(cap=30.0, window=0, sink=0, slope=None, span=None):
    return vsa2.vsa2_scores(cap, window, sink, slope, span)


def assign(c=None, table=FAKE, refs=FAKE, length=FAKE, source=None, drop=None, count=None, room=None, ws=FAKE, ws_bytes=BIG):
    return NAME[vsa2.vsa2_cache_assign(c or cache(), table, refs, length, source, drop, count, room, ws, ws_bytes)]


def copy(a=None, b=None, n=3, index=FAKE, start=FAKE, count=None):
    return NAME[vsa2.vsa2_cache_copy(a or cache(), b or cache(), n, index, start, count)]


def shared(p=None, c=None, dtype=1, heads=8, n=3, q=rows(), plen=FAKE, length=FAKE, o=rows(), lse=FAKE, ws=FAKE, ws_bytes=BIG):
    return NAME[vsa2.vsa2_attn_cache_shared(p or cache(batch=2), c or cache(), dtype, heads, n, q, plen, length, None, 0, o, lse,
                                            ws, ws_bytes)]


def scored(c=None, s=scores(), dtype=1, heads=8, n=3, q=rows(), length=FAKE, o=rows(), lse=FAKE, ws=FAKE, ws_bytes=BIG):
    return NAME[vsa2.vsa2_attn_cache_scored(c or cache(), s, dtype, heads, n, q, length, None, 0, o, lse, ws, ws_bytes)]


CACHE_BAD = [
    ("VSA2_ERR_SHAPE", dict(batch=0)), ("VSA2_ERR_SHAPE", dict(heads_kv=0)), ("VSA2_ERR_SHAPE", dict(pages=0)),
    ("VSA2_ERR_SHAPE", dict(max_pages=0)), ("VSA2_ERR_SHAPE", dict(table_heads=2)),
    ("VSA2_ERR_UNSUPPORTED", dict(head_dim=96)), ("VSA2_ERR_UNSUPPORTED", dict(max_pages=(1 << 24) + 1)),
    ("VSA2_ERR_NULL", dict(pool=None)), ("VSA2_ERR_NULL", dict(table=None)), ("VSA2_ERR_ALIGN", dict(pool=FAKE + 128)),
]


@pytest.mark.parametrize("want,kw", CACHE_BAD)
def test_calls_refuse_a_bad_cache(want, kw):
    assert assign(c=cache(**kw)) == want
    assert scored(c=cache(**kw)) == want
    assert shared(c=cache(**kw)) == want
    # the other cache of a call: of other sizes it does not fit this one
    assert copy(a=cache(**kw)) in (want, "VSA2_ERR_SHAPE") and copy(b=cache(**kw)) in (want, "VSA2_ERR_SHAPE")
    assert shared(p=cache(**dict(batch=2) | kw)) in (want, "VSA2_ERR_SHAPE")


@pytest.mark.parametrize("want,kw", [
    ("VSA2_ERR_SHAPE", dict(c=cache(table_heads=4))),                    # lists per KV head
    ("VSA2_ERR_NULL", dict(table=None)), ("VSA2_ERR_NULL", dict(refs=None)), ("VSA2_ERR_NULL", dict(length=None)),
    ("VSA2_ERR_VALUE", dict(table=FAKE + 256)),                          # not the cache's
    ("VSA2_ERR_ALIGN", dict(refs=FAKE + 4)), ("VSA2_ERR_ALIGN", dict(ws=FAKE + 16)),
    ("VSA2_ERR_WORKSPACE", dict(ws=None)), ("VSA2_ERR_WORKSPACE", dict(ws_bytes=512)),
    ("VSA2_ERR_UNSUPPORTED", dict(c=cache(batch=1 << 20, max_pages=1 << 12))),
    ("VSA2_ERR_UNSUPPORTED", dict(c=cache(batch=1 << 24, max_pages=1))),
    ("VSA2_ERR_UNSUPPORTED", dict(c=cache(heads_kv=32769))),
])
def test_assign_refuses(want, kw):
    assert assign(**kw) == want


@pytest.mark.parametrize("want,kw", [
    ("VSA2_ERR_SHAPE", dict(n=-1)), ("VSA2_ERR_NULL", dict(index=None)), ("VSA2_ERR_NULL", dict(start=None)),
    ("VSA2_ERR_SHAPE", dict(b=cache(batch=2))), ("VSA2_ERR_SHAPE", dict(b=cache(heads_kv=2))),
    ("VSA2_ERR_SHAPE", dict(a=cache(head_dim=64))),
    ("VSA2_ERR_UNSUPPORTED", dict(n=2 ** 31 - 1, a=cache(batch=1 << 20), b=cache(batch=1 << 20))),
])
def test_copy_refuses(want, kw):
    assert copy(**kw) == want


ATTN_BAD = [
    ("VSA2_ERR_DTYPE", dict(dtype=-1)), ("VSA2_ERR_SHAPE", dict(n=-1)), ("VSA2_ERR_SHAPE", dict(heads=6)),
    ("VSA2_ERR_SHAPE", dict(heads=0)), ("VSA2_ERR_NULL", dict(q=None)), ("VSA2_ERR_NULL", dict(o=None)),
    ("VSA2_ERR_NULL", dict(length=None)), ("VSA2_ERR_NULL", dict(lse=None)), ("VSA2_ERR_SHAPE", dict(o=rows(t=0))),
    ("VSA2_ERR_ALIGN", dict(q=rows(h=130))), ("VSA2_ERR_UNSUPPORTED", dict(n=1 << 30)),
]


@pytest.mark.parametrize("want,kw", ATTN_BAD + [
    ("VSA2_ERR_NULL", dict(plen=None)), ("VSA2_ERR_SHAPE", dict(p=cache(batch=3))), ("VSA2_ERR_SHAPE", dict(p=cache(batch=8))),
    ("VSA2_ERR_SHAPE", dict(p=cache(heads_kv=2))), ("VSA2_ERR_SHAPE", dict(p=cache(head_dim=64))),
    ("VSA2_ERR_UNSUPPORTED", dict(p=cache(batch=1), c=cache(batch=1 << 16, heads_kv=1), n=1 << 13, heads=4)),
    ("VSA2_ERR_WORKSPACE", dict(ws=None)), ("VSA2_ERR_WORKSPACE", dict(ws_bytes=1024)), ("VSA2_ERR_ALIGN", dict(ws=FAKE + 16)),
])
def test_shared_refuses(want, kw):
    assert shared(**kw) == want


@pytest.mark.parametrize("want,kw", ATTN_BAD + [
    ("VSA2_ERR_NULL", dict(s=None)), ("VSA2_ERR_VALUE", dict(s=scores(cap=-1.0))),
    ("VSA2_ERR_VALUE", dict(s=scores(cap=float("nan")))), ("VSA2_ERR_VALUE", dict(s=scores(cap=float("inf")))),
    ("VSA2_ERR_VALUE", dict(s=scores(cap=2.0 ** 21))), ("VSA2_ERR_VALUE", dict(s=scores(cap=2.0 ** -21))),
    ("VSA2_ERR_VALUE", dict(s=scores(window=-1))), ("VSA2_ERR_VALUE", dict(s=scores(sink=-1))),
    ("VSA2_ERR_WORKSPACE", dict(c=cache(max_pages=400), ws=None)), ("VSA2_ERR_ALIGN", dict(c=cache(max_pages=400), ws=FAKE + 16)),
])
def test_scored_refuses(want, kw):
    assert scored(**kw) == want


def test_workspaces_and_nothing_to_do():
    c = cache(max_pages=400)
    st, need = vsa2.vsa2_attn_cache_shared_workspace(cache(batch=2, max_pages=400), c, 8, 1)
    assert NAME[st] == "VSA2_OK" and need > 0 and need % 256 == 0
    assert vsa2.vsa2_attn_cache_shared_workspace(cache(batch=2), c, 8, 0) == (0, 0)
    st, need = vsa2.vsa2_attn_cache_scored_workspace(c, scores(), 8, 1)
    assert NAME[st] == "VSA2_OK" and need > 0 and need % 256 == 0
    # a window needs no more than its pages
    assert vsa2.vsa2_attn_cache_scored_workspace(cache(max_pages=4000), scores(window=100), 8, 1)[1] < need
    assert vsa2.vsa2_attn_cache_scored_workspace(c, scores(window=2 ** 31 - 1, sink=2 ** 31 - 1), 8, 1)[1] == need
    st, need = vsa2.vsa2_cache_assign_workspace(c)
    assert NAME[st] == "VSA2_OK" and need > 4 * 4 * 400 and need % 256 == 0
    assert NAME[vsa2.vsa2_cache_assign_workspace(cache(table_heads=4))[0]] == "VSA2_ERR_SHAPE"
    assert NAME[vsa2.vsa2_attn_cache_scored_workspace(c, None, 8, 1)[0]] == "VSA2_ERR_NULL"
    assert NAME[vsa2.vsa2_attn_cache_shared_workspace(None, c, 8, 1)[0]] == "VSA2_ERR_NULL"
    # no tokens: nothing is looked at beyond the sizes
    assert shared(n=0, q=None, plen=None, length=None, o=None, lse=None, ws=None, ws_bytes=0) == "VSA2_OK"
    assert scored(n=0, q=None, length=None, o=None, lse=None, ws=None, ws_bytes=0) == "VSA2_OK"
    assert copy(n=0, index=None, start=None) == "VSA2_OK"
    assert NAME[vsa2.vsa2_cache_copy(None, cache(), 1, FAKE, FAKE, None)] == "VSA2_ERR_NULL"
    assert ctypes.sizeof(vsa2.vsa2_scores) == 32


def test_helpers_refuse():
    torch = pytest.importorskip("torch")

    class Fake:
        c, table, device = cache(), torch.zeros(4, 6, dtype=torch.int32), -1

    ints = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="table: expected"):
        vsa2.cache_assign(Fake, torch.zeros(10, dtype=torch.int32), ints)
    with pytest.raises(ValueError, match="index: expected"):
        vsa2.cache_copy(Fake, Fake, ints, ints)
    with pytest.raises(ValueError, match="index: expected"):
        vsa2.cache_copy(Fake, Fake, torch.zeros(4, 3, dtype=torch.int32), ints)
    q = torch.zeros(4, 8, 3, 128)
    with pytest.raises(ValueError, match="q: expected"):
        vsa2.attn_cache_shared(Fake, Fake, q, ints, ints)
    with pytest.raises(ValueError, match="q: expected"):
        vsa2.attn_cache_scored(Fake, q, ints)
