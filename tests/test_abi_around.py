"""What the operators around the attention refuse, on the host: every call here
fails (or has nothing to do) before any device work, so no pointer is followed."""
import ctypes

import pytest

vsa2 = pytest.importorskip("paper_2609_32882_amd")

FAKE, MISALIGNED = 0x10000, 0x10008
BIG = 1 << 40
NAME = vsa2.STATUS_NAMES


def rows(ptr=FAKE, b=1 << 20, h=128, t=1024):
    return vsa2.vsa2_rows(ptr, b, h, t)


def rope(axis=(44, 42, 42), rows=(8, 16, 16), table=(FAKE, FAKE, FAKE), origin=None, pairing=0):
    r = vsa2.vsa2_rope(pairing=pairing, origin=origin)
    for i in range(3):
        r.axis[i], r.rows[i], r.table[i] = axis[i], rows[i], table[i]
    return r


def problem(**kw):
    p = vsa2.make_problem(2, 4, 2, 128, 8, 16, 16)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def forward(p=None, r=None, eps=1e-6, q_in=None, q_gain=FAKE, q=FAKE, k_in=None, k_gain=None, k=None, v_in=None, v=None):
    return NAME[vsa2.vsa2_qk_norm_rope(p or problem(), r, eps, q_in, q_gain, q, k_in, k_gain, k, v_in, v, None)]


@pytest.mark.parametrize("want,kw", [
    ("VSA2_ERR_NULL", dict(q_in=None)),                                  # an output without its rows
    ("VSA2_ERR_NULL", dict(q_in=rows(), q=None)),
    ("VSA2_ERR_NULL", dict(q_in=rows(ptr=None))),
    ("VSA2_ERR_ALIGN", dict(q_in=rows(ptr=MISALIGNED))),
    ("VSA2_ERR_ALIGN", dict(q_in=rows(), q=MISALIGNED)),
    ("VSA2_ERR_ALIGN", dict(q_in=rows(h=132))),                          # 264 bytes in bf16
    ("VSA2_ERR_SHAPE", dict(q_in=rows(t=-128))),
    ("VSA2_ERR_VALUE", dict(q_in=rows(), eps=-1e-6)),
    ("VSA2_ERR_VALUE", dict(q_in=rows(), eps=float("nan"))),
    ("VSA2_ERR_VALUE", dict(q_in=rows(), eps=float("inf"))),
    ("VSA2_ERR_VALUE", dict(q_in=rows(), eps=0.0)),                      # a gain without the norm
    ("VSA2_ERR_VALUE", dict(q_in=rows(), r=rope(pairing=2))),
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), r=rope(axis=(44, 42, 44)))),    # 130 of 128 elements
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), r=rope(axis=(43, 42, 42)))),
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), r=rope(axis=(-2, 42, 42)))),
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), r=rope(axis=(44, 42, 40), pairing=1))),   # 126: halves need 8
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), r=rope(rows=(8, 15, 16)))),     # a table shorter than the grid
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), r=rope(rows=(8, 0, 16), origin=FAKE))),
    ("VSA2_ERR_NULL", dict(q_in=rows(), r=rope(table=(FAKE, None, FAKE)))),
    ("VSA2_ERR_ALIGN", dict(q_in=rows(), r=rope(table=(FAKE, FAKE + 4, FAKE)))),
    ("VSA2_ERR_UNSUPPORTED", dict(q_in=rows(), p=problem(head_dim=96))),
    ("VSA2_ERR_UNSUPPORTED", dict(q_in=rows(), p=problem(T=8192, H=1024, W=1024, Bt=8, Bh=8, Bw=8))),
    ("VSA2_ERR_DTYPE", dict(q_in=rows(), p=problem(dtype=5))),
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), p=problem(T=0))),
])
def test_norm_rope_refuses(want, kw):
    assert forward(**kw) == want


def test_norm_rope_with_nothing_to_do():
    assert forward(q=None) == "VSA2_OK"
    # the strides of an axis with one entry are not looked at
    p = vsa2.make_problem(1, 1, 1, 128, 1, 1, 1, 1, 1, 1, 1, 1, 1)
    assert forward(p=p, q_in=rows(b=3, h=-5, t=7), q=MISALIGNED) == "VSA2_ERR_ALIGN"
    assert forward(p=p, q_in=rows(b=3, h=-5, t=7), q=None) == "VSA2_ERR_NULL"


def backward(p=None, r=None, eps=1e-6, q_in=None, q_gain=None, dq=FAKE, dq_in=None, dq_gain=FAKE, dk=None, dk_gain=None,
             ws=FAKE, ws_bytes=BIG):
    return NAME[vsa2.vsa2_qk_norm_rope_bwd(p or problem(), r, eps, q_in, q_gain, dq, dq_in, dq_gain, None, None, dk, None,
                                           dk_gain, None, None, ws, ws_bytes, None)]


@pytest.mark.parametrize("want,kw", [
    ("VSA2_ERR_NULL", dict(dq_in=rows())),                               # the norm needs x
    ("VSA2_ERR_NULL", dict(q_in=rows())),
    ("VSA2_ERR_NULL", dict(q_in=rows(), dq_in=rows(), dq=None)),
    ("VSA2_ERR_NULL", dict(q_in=rows(), dq_in=rows(), dk_gain=FAKE)),    # a gain's gradient without its rows
    ("VSA2_ERR_SHAPE", dict(q_in=rows(), dq_in=rows(t=0))),              # written rows must not overlap
    ("VSA2_ERR_ALIGN", dict(q_in=rows(), dq_in=rows(), dq=MISALIGNED)),
    ("VSA2_ERR_VALUE", dict(q_in=rows(), dq_in=rows(), eps=0.0)),
    ("VSA2_ERR_WORKSPACE", dict(q_in=rows(), dq_in=rows(), ws=None)),
    ("VSA2_ERR_WORKSPACE", dict(q_in=rows(), dq_in=rows(), ws_bytes=1023)),
    ("VSA2_ERR_ALIGN", dict(q_in=rows(), dq_in=rows(), ws=FAKE + 16)),
    ("VSA2_ERR_VALUE", dict(q_in=rows(), dq_in=rows(), r=rope(pairing=-1))),
])
def test_norm_rope_bwd_refuses(want, kw):
    assert backward(**kw) == want


def cache(**kw):
    c = vsa2.vsa2_cache(2, 4, 128, 10, 6, 1, FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


CACHE_BAD = [
    ("VSA2_ERR_SHAPE", dict(batch=0)), ("VSA2_ERR_SHAPE", dict(heads_kv=0)), ("VSA2_ERR_SHAPE", dict(pages=0)),
    ("VSA2_ERR_SHAPE", dict(max_pages=0)), ("VSA2_ERR_SHAPE", dict(table_heads=2)),
    ("VSA2_ERR_UNSUPPORTED", dict(head_dim=96)), ("VSA2_ERR_UNSUPPORTED", dict(max_pages=(1 << 24) + 1)),
    ("VSA2_ERR_NULL", dict(pool=None)), ("VSA2_ERR_NULL", dict(table=None)), ("VSA2_ERR_ALIGN", dict(pool=FAKE + 128)),
]


@pytest.mark.parametrize("want,kw", CACHE_BAD)
def test_cache_calls_refuse_a_bad_cache(want, kw):
    c = cache(**kw)
    assert NAME[vsa2.vsa2_cache_write(c, 1, 3, rows(), rows(), FAKE, None)] == want
    assert NAME[vsa2.vsa2_cache_read(c, 1, 3, rows(), rows(), FAKE, None)] == want
    assert NAME[vsa2.vsa2_attn_cache(c, 1, 8, 3, rows(), FAKE, None, 0, rows(), FAKE, FAKE, BIG)] == want


@pytest.mark.parametrize("want,kw", [
    ("VSA2_ERR_DTYPE", dict(dtype=2)), ("VSA2_ERR_SHAPE", dict(n=-1)), ("VSA2_ERR_NULL", dict(k=None)),
    ("VSA2_ERR_NULL", dict(v=rows(ptr=None))), ("VSA2_ERR_NULL", dict(start=None)),
    ("VSA2_ERR_ALIGN", dict(k=rows(ptr=MISALIGNED))), ("VSA2_ERR_ALIGN", dict(v=rows(t=1025))),
    ("VSA2_ERR_SHAPE", dict(k=rows(b=-1024))), ("VSA2_ERR_UNSUPPORTED", dict(n=2 ** 31 - 1, c=cache(batch=1 << 20))),
])
def test_cache_copies_refuse(want, kw):
    a = dict(c=cache(), dtype=1, n=3, k=rows(), v=rows(), start=FAKE) | kw
    for call in (vsa2.vsa2_cache_write, vsa2.vsa2_cache_read):
        assert NAME[call(a["c"], a["dtype"], a["n"], a["k"], a["v"], a["start"], None)] == want
    # only the read writes its rows
    assert NAME[vsa2.vsa2_cache_read(cache(), 1, 3, rows(h=0), rows(), FAKE, None)] == "VSA2_ERR_SHAPE"


@pytest.mark.parametrize("want,kw", [
    ("VSA2_ERR_DTYPE", dict(dtype=-1)), ("VSA2_ERR_SHAPE", dict(n=-1)), ("VSA2_ERR_SHAPE", dict(heads=6)),
    ("VSA2_ERR_SHAPE", dict(heads=0)), ("VSA2_ERR_NULL", dict(q=None)), ("VSA2_ERR_NULL", dict(o=None)),
    ("VSA2_ERR_NULL", dict(length=None)), ("VSA2_ERR_NULL", dict(lse=None)), ("VSA2_ERR_SHAPE", dict(o=rows(t=0))),
    ("VSA2_ERR_ALIGN", dict(q=rows(h=130))), ("VSA2_ERR_UNSUPPORTED", dict(n=1 << 30)),
])
def test_attn_cache_refuses(want, kw):
    a = dict(dtype=1, heads=8, n=3, q=rows(), o=rows(), length=FAKE, lse=FAKE) | kw
    assert NAME[vsa2.vsa2_attn_cache(cache(), a["dtype"], a["heads"], a["n"], a["q"], a["length"], None, 0, a["o"],
                                     a["lse"], FAKE, BIG)] == want


def test_attn_cache_workspace():
    c = cache(max_pages=400)
    st, need = vsa2.vsa2_attn_cache_workspace(c, 8, 1)
    assert NAME[st] == "VSA2_OK" and need > 0 and need % 256 == 0
    args = (c, 1, 8, 1, rows(), FAKE, None, 0, rows(), FAKE)
    assert NAME[vsa2.vsa2_attn_cache(*args, None, 0)] == "VSA2_ERR_WORKSPACE"
    assert NAME[vsa2.vsa2_attn_cache(*args, FAKE, need - 1)] == "VSA2_ERR_WORKSPACE"
    assert NAME[vsa2.vsa2_attn_cache(*args, FAKE + 16, need)] == "VSA2_ERR_ALIGN"
    assert vsa2.vsa2_attn_cache_workspace(c, 8, 0) == (0, 0)
    # no tokens: nothing is looked at beyond the sizes
    assert NAME[vsa2.vsa2_attn_cache(c, 1, 8, 0, None, None, None, 0, None, None, None, 0)] == "VSA2_OK"
    assert NAME[vsa2.vsa2_cache_write(c, 1, 0, None, None, None, None)] == "VSA2_OK"


def test_null_structures_and_page_bytes():
    assert NAME[vsa2.vsa2_cache_write(None, 1, 1, rows(), rows(), FAKE, None)] == "VSA2_ERR_NULL"
    assert NAME[vsa2.vsa2_attn_cache(None, 1, 8, 1, rows(), FAKE, None, 0, rows(), FAKE, FAKE, BIG)] == "VSA2_ERR_NULL"
    assert NAME[vsa2.vsa2_qk_norm_rope(None, None, 0.0, rows(), None, FAKE, None, None, None, None, None)] == "VSA2_ERR_NULL"
    assert vsa2.vsa2_cache_page_bytes(128) == (0, 16512) and vsa2.vsa2_cache_page_bytes(64) == (0, 8320)
    assert NAME[vsa2.vsa2_cache_page_bytes(80)[0]] == "VSA2_ERR_UNSUPPORTED"
    assert ctypes.sizeof(vsa2.vsa2_rows) == 32 and ctypes.sizeof(vsa2.vsa2_cache) == 40 and \
        ctypes.sizeof(vsa2.vsa2_rope) == 64


def test_helpers_refuse():
    torch = pytest.importorskip("torch")
    cpu = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError, match="pool"):
        vsa2.KVCache(torch.zeros(2, 2, 100, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="on the GPU"):
        vsa2.qk_norm_rope(vsa2.make_problem(1, 2, 2, 64, 1, 1, 3, 1, 1, 1, 1, 1, 1, vsa2.VSA2_F32), cpu)
    with pytest.raises(KeyError):
        vsa2.Rope((64, 0, 0), [None] * 3, pairing="other")
