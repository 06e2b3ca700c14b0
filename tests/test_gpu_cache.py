"""The 8-bit cache: writes against the plain quantisation bit by bit, reads
exactly, at positions that start and end inside pages."""
import pytest
import torch

import around_reference as ref
import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# batch, heads, D, n, max_pages, start per sequence, count per sequence (None: n), lists per head, dtype
CASES = [
    (3, 2, 128, 1, 2, [0, 63, 64], None, False, "bf16"),
    (2, 2, 64, 1, 3, [17, 130], [1, 0], True, "f32"),
    (1, 3, 128, 64, 1, [0], None, False, "bf16"),
    (2, 1, 128, 65, 3, [63, 1], None, False, "f32"),
    (2, 2, 64, 66, 4, [63, 127], [66, 5], True, "bf16"),
    (1, 2, 64, 200, 4, [50], None, False, "f32"),
    (2, 2, 128, 150, 4, [64, 3], [129, 150], False, "bf16"),
    (2, 1, 64, 100, 2, [-30, 90], None, False, "bf16"),       # positions outside the list on both sides
    (2, 2, 128, 9, 2, [5, 2000000000], [-4, 99], False, "bf16"),
]
IDS = ["n%d-D%d-%s%s" % (c[3], c[2], c[8], "-lists" if c[7] else "") for c in CASES]


def make(case, seed=0):
    batch, heads, D, n, max_pages, start, count, lists, dtype = case
    g = torch.Generator().manual_seed(seed)
    pages = batch * max_pages + 2
    pool = torch.randint(0, 256, (pages, heads, 128 * D + 128), generator=g, dtype=torch.uint8)
    order = torch.randperm(pages, generator=g)[:batch * max_pages].to(torch.int32)
    table = order.view(batch, max_pages)
    if lists:
        table = torch.stack([order.roll(h).view(batch, max_pages) for h in range(heads)], 1).contiguous()
    kv = torch.randn(batch, n, 2 * heads, D, generator=g) * torch.randn(batch, n, 2 * heads, 1, generator=g).mul(3).exp()
    kv = kv.to(DT[dtype])
    return (pool, table, kv, torch.tensor(start, dtype=torch.int32),
            None if count is None else torch.tensor(count, dtype=torch.int32))


def gpu(t):
    return None if t is None else t.cuda()


def heads_first(kv, heads):
    return [x.transpose(1, 2) for x in kv.split(heads, 2)]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_write_and_read(case):
    batch, heads, D, n, *_ = case
    pool, table, kv, start, count = make(case)
    k, v = heads_first(kv, heads)
    dev = pool.cuda()
    cache = vsa2.KVCache(dev, table.cuda())
    vsa2.cache_write(cache, *heads_first(kv.cuda(), heads), start.cuda(), gpu(count))
    want = ref.write_reference(pool.clone(), table, k, v, start, count)
    assert torch.equal(dev.cpu(), want)                # every byte, the untouched ones too
    for dtype in (torch.bfloat16, torch.float32):
        got = vsa2.cache_read(cache, n, start.cuda(), gpu(count), dtype=dtype)
        for a, b in zip(got, ref.read_reference(want, table, n, start, count, D, heads)):
            assert torch.equal(a.double().cpu(), b.to(dtype).double())   # a code times a power is exact in bf16


def test_values_of_every_kind():
    """Rounding ties, the smallest codes, zeros, values that are not finite."""
    D = 64
    g = torch.Generator().manual_seed(5)
    rows = torch.randn(64, D, generator=g)
    # the middle between neighbouring codes, and its neighbours on both sides
    grid = ref.VALUES[:127]
    mid = ((grid[1:] + grid[:-1]) / 2).float()
    rows[0, :63], rows[0, 63] = mid[:63], 448.0
    rows[1, :63], rows[1, 63] = mid[63:126], 448.0
    rows[2] = torch.nextafter(rows[0], torch.full((D,), 1e9))
    rows[2, 63] = 448.0
    rows[3] = -torch.nextafter(rows[1], torch.zeros(D))
    rows[4] = 0.0
    rows[5] = -0.0
    rows[6, 3], rows[6, 4], rows[6, 5] = float("nan"), float("inf"), -float("inf")
    rows[7] = float("nan")
    rows[8] = rows[8] * 1e-38                           # subnormal in fp32
    rows[9] = rows[9] * 1e-25
    rows[10] = rows[10] * 2.0 ** 120
    rows[11, :2] = torch.tensor([3.3e38, -2.0 ** 127])
    rows[12] = 448.0 * 1.0000001
    rows[13] = torch.ldexp(torch.tensor(448.0), torch.tensor(-40))
    rows[14] = torch.ldexp(torch.tensor(449.0), torch.tensor(7))
    x = rows.view(1, 1, 64, D)
    pool = torch.zeros(1, 1, 128 * D + 128, dtype=torch.uint8)
    table = torch.zeros(1, 1, dtype=torch.int32)
    start = torch.zeros(1, dtype=torch.int32)
    dev = pool.cuda()
    cache = vsa2.KVCache(dev, table.cuda())
    vsa2.cache_write(cache, x.cuda(), (-x).contiguous().cuda(), start.cuda())
    want = ref.write_reference(pool.clone(), table, x, -x, start, None)
    got = dev.cpu()
    same = got == want
    # a NaN's sign is not kept: either NaN code will do
    nan = ((got & 0x7f) == 0x7f) & ((want & 0x7f) == 0x7f)
    nan[..., 128 * D:] = False
    assert (same | nan).all()
    k, v = vsa2.cache_read(cache, 64, start.cuda(), dtype=torch.float32)
    for a, b in zip((k, v), ref.read_reference(want, table, 64, start, None, D, 1)):
        a, b = a.double().cpu(), b.float().double()
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def test_pages_outside_the_pool_are_skipped():
    case = (2, 2, 64, 150, 3, [0, 0], None, False, "bf16")
    pool, table, kv, start, count = make(case)
    table[0, 1], table[1, 0], table[1, 2] = -1, pool.shape[0], 2 ** 31 - 1
    dev = pool.cuda()
    cache = vsa2.KVCache(dev, table.cuda())
    vsa2.cache_write(cache, *heads_first(kv.cuda(), 2), start.cuda())
    want = ref.write_reference(pool.clone(), table, *heads_first(kv, 2), start, None)
    assert torch.equal(dev.cpu(), want)
    got = vsa2.cache_read(cache, 150, start.cuda())
    for a, b in zip(got, ref.read_reference(want, table, 150, start, None, 64, 2)):
        assert torch.equal(a.double().cpu(), b)


def test_a_row_keeps_four_bits():
    """Reading back is within 2^-4 of a value down to 2^-13 of the row's largest."""
    x = torch.randn(1, 2, 64, 128, generator=torch.Generator().manual_seed(1))
    table, start = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    cache = vsa2.KVCache.empty(table, 1, 2, 128)
    vsa2.cache_write(cache, x.cuda(), x.cuda(), start)
    k, v = vsa2.cache_read(cache, 64, start, dtype=torch.float32)
    assert torch.equal(k, v)
    far = (k.cpu() - x).abs()
    top = x.abs().amax(-1, keepdim=True)
    assert (far <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -17 * top)).all()
    # written again, the values read are stored as they are
    vsa2.cache_write(cache, k, v, start)
    assert torch.equal(vsa2.cache_read(cache, 64, start, dtype=torch.float32)[0], k)


def test_strided_outputs_guards_and_nothing_to_do():
    case = (2, 2, 128, 70, 3, [10, 60], [70, 33], False, "bf16")
    pool, table, kv, start, count = make(case)
    cache = vsa2.KVCache(pool.cuda(), table.cuda())
    vsa2.cache_write(cache, *heads_first(kv.cuda(), 2), start.cuda(), count.cuda())
    plain = vsa2.cache_read(cache, 70, start.cuda(), count.cuda())
    buf = torch.full((2, 72, 6, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    out = [buf[:, 1:71, i:i + 2].transpose(1, 2) for i in (1, 3)]
    vsa2.cache_read(cache, 70, start.cuda(), count.cuda(), out=out)
    for a, b in zip(out, plain):
        assert torch.equal(a, b)
    assert (buf[:, 0] == 7).all() and (buf[:, 71] == 7).all() and (buf[:, :, 0] == 7).all() and (buf[:, :, 5] == 7).all()
    before = cache.pool.clone()
    none = torch.empty(2, 2, 0, 128, dtype=torch.bfloat16, device="cuda")
    vsa2.cache_write(cache, none, none, start.cuda())
    assert torch.equal(cache.pool, before) and vsa2.cache_read(cache, 0, start.cuda())[0].shape == (2, 2, 0, 128)
