"""Caps that the scored attention's helper takes and refuses: 0 is no cap, and a number that fp32 has as
0 is not that."""
import pytest
import torch

import paper_2609_32882_amd as vsa2

pytestmark = pytest.mark.gpu


def call(cap):
    cache = vsa2.KVCache.empty(torch.zeros(1, 1, dtype=torch.int32).cuda(), 1, 1, 64)
    q, one = torch.randn(1, 1, 4, 64, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    vsa2.cache_write(cache, q, q, torch.zeros(1, dtype=torch.int32).cuda())
    return vsa2.attn_cache_scored(cache, q, one, cap=cap)[0]


@pytest.mark.parametrize("cap", [1e-50, -1e-50, 5e-324, 1e-40, -1e-40, 2.0 ** -21, -1.0, 2.0 ** 20 * 1.001, 1e300,
                                 float("inf"), float("nan")])
def test_refused(cap):
    with pytest.raises(vsa2.Vsa2Error, match="VSA2_ERR_VALUE"):
        call(cap)


@pytest.mark.parametrize("cap", [0, 0.0, -0.0, 2.0 ** -20, 30, 2.0 ** 20])
def test_taken(cap):
    assert torch.isfinite(call(cap)).all()
