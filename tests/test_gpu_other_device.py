"""A cache or a rotation made on one GPU and used while another is current: refused, since
its addresses are the first one's.  One GPU is enough: the number it was made on is planted."""
import pytest
import torch

import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu


def test_a_cache_of_another_gpu_is_refused():
    table = torch.zeros(1, 1, dtype=torch.int32).cuda()
    cache = vsa2.KVCache.empty(table, 1, 1, 64)
    x = torch.randn(1, 1, 4, 64, device="cuda")
    start, length = torch.zeros(1, dtype=torch.int32).cuda(), torch.full((1,), 4, dtype=torch.int32).cuda()
    vsa2.cache_write(cache, x, x, start)
    before = cache.pool.clone()
    assert cache.device == torch.cuda.current_device()
    cache.device += 1
    for call in (lambda: vsa2.cache_write(cache, -x, -x, start), lambda: vsa2.cache_read(cache, 4, start),
                 lambda: vsa2.attn_cache(cache, x, length)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert torch.equal(cache.pool, before)
    cache.device -= 1
    assert torch.isfinite(vsa2.attn_cache(cache, x, length)[0]).all()


def test_a_rotation_of_another_gpu_is_refused():
    p = vsa2.make_problem(1, 1, 1, 64, 1, 1, 8, 1, 1, 1, 1, 1, 1, vsa2.VSA2_F32)
    x = torch.randn(1, 1, 8, 64, device="cuda")
    origin = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    for rope in (vsa2.Rope((0, 0, 64), (None, None, vsa2.rope_table(8, 64))), vsa2.Rope((0, 0, 0), (None,) * 3, origin)):
        assert rope.device == torch.cuda.current_device()
        rope.device += 1
        with pytest.raises(ValueError, match="current device"):
            vsa2.qk_norm_rope(p, x, rope=rope)
        with pytest.raises(ValueError, match="current device"):
            vsa2.qk_norm_rope_bwd(p, x, rope=rope)
    assert vsa2.Rope((0, 0, 0), (None,) * 3).device == -1        # nothing of any GPU
