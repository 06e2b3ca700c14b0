"""The bias by distance where a token's own position ends a page: there a page's positions are
all on one side of every row's own, and the token itself is among them, with no bias at all.

Slopes of 2^10 and more leave one token of weight 1, whose score is the lse.  A positive slope
leaves the row's own, with nothing of the bias in it; the bound is that of
test_gpu_attn_cache_scored.py's slopes at their ends."""
import pytest
import torch

import paging_reference as pref
from test_gpu_attn_cache import make
from test_gpu_attn_cache_scored import run

pytestmark = pytest.mark.gpu

# tokens of the call and the list's length: the first token is the last of its page; one row a head, tiles of 16,
# 128 rows a workgroup
CALLS = [(1, 64), (1, 128), (1, 256), (20, 83), (20, 147), (140, 203), (140, 267)]


@pytest.mark.parametrize("n,length", CALLS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [0.0, 30.0, 2.0 ** 20])
@pytest.mark.parametrize("D", [64, 128])
def test_the_own_position_at_a_pages_end(n, length, dtype, cap, D):
    case = (2, 4, 2, D, n, 5, [length, length], None, True, False, dtype)
    x = make(case)
    opt = dict(cap=cap, slope=torch.tensor([2.0 ** 10, 2.0 ** 20, 2.0 ** 90, -2.0 ** 90]), window=0, sink=0, span=None)
    o, lse = (y.double().cpu() for y in run(case, x[0], x, opt))
    wo, wl, _, logit = pref.scored_reference(*x[:5], case[8], **opt)
    # one term: the weight's fp16 (2^-11) and the result's rounding, or three bf16 terms of the weight, their
    # products' sum, the reciprocal and its product, some 2^-24 each
    step = 2.0 ** -8 + 2.0 ** -10 if dtype == "bf16" else 2.0 ** -21
    assert ((o - wo).abs() <= step * wo.abs()).all()
    # own scores: the product's error, that of log2 e and back and of the cap; far ones: the distance's product
    delta = 2.0 ** -20 * logit[..., 0] + 2.0 ** -21 * (1 + wl.abs() + min(cap, 64.0))
    assert ((lse - wl).abs() <= delta).all(), ((lse - wl).abs() - delta).max()


@pytest.mark.parametrize("n,length,span", [(1, 65, None), (1, 129, None), (140, 204, (128, 204))])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_own_position_before_a_page(n, length, span, dtype):
    """The own position is a page's first, and pages that begin behind those of a tile's rows."""
    case = (1, 4, 2, 64, n, 5, [length], None, False, False, dtype)
    x = make(case)
    opt = dict(cap=0.0, slope=torch.tensor([2.0 ** 10, 2.0 ** 20, 2.0 ** 90, 2.0 ** 60]), window=0, sink=0, span=None)
    if span:
        opt["span"] = torch.tensor(span, dtype=torch.int32).expand(1, n, 2).contiguous()
    o, lse = (y.double().cpu() for y in run(case, x[0], x, opt))
    wo, wl, _, logit = pref.scored_reference(*x[:5], case[8], **opt)
    step = 2.0 ** -8 + 2.0 ** -10 if dtype == "bf16" else 2.0 ** -21
    assert ((o - wo).abs() <= step * wo.abs()).all()
    assert ((lse - wl).abs() <= 2.0 ** -20 * logit[..., 0] + 2.0 ** -21 * (1 + wl.abs())).all()
