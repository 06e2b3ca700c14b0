"""The scored attention where pairs of row tiles share a page's codes: many lists, 17 to 32 rows a head."""
import pytest

import paging_reference as pref
from test_gpu_attn_cache import make
from test_gpu_attn_cache_scored import check, options, run

pytestmark = pytest.mark.gpu

LENGTHS = [1, 64, 130, 77, 0, 200, 63, 65, 128, 20, 21, 190, 100, 45, 129, 33]
COUNTS = [20, 20, 7, 20, 20, 17, 16, 20, 0, 20, 1, 20, 20, 15, 20, 20]

# 64 lists of two tiles: in one launch (pages up to 32), and in pieces (128 pages, of which lists fill a few)
CASES = [
    ((16, 4, 4, 64, 20, 4, LENGTHS, None, True, False, "bf16"), 30.0, True, 40, 3, "holes"),
    ((16, 4, 4, 128, 20, 4, LENGTHS, COUNTS, False, False, "bf16"), 30.0, True, 0, 0, "doc"),
    ((16, 4, 4, 64, 20, 4, LENGTHS, COUNTS, True, False, "f32"), 20.0, True, 0, 70, "holes"),
    ((16, 4, 4, 128, 20, 128, LENGTHS[:-1] + [900], COUNTS, True, False, "bf16"), 30.0, True, 0, 0, "holes"),
    ((16, 4, 4, 64, 20, 128, LENGTHS[:-1] + [900], None, False, False, "bf16"), 0.0, True, 0, 5, "holes"),
    ((16, 4, 4, 64, 20, 128, LENGTHS[:-1] + [900], COUNTS, False, False, "f32"), 20.0, False, 0, 0, "holes"),
]


@pytest.mark.parametrize("case,cap,slope,window,sink,span", CASES,
                         ids=["D%d-%d pages-%s" % (c[0][3], c[0][5], c[0][10]) for c in CASES])
def test_matches_the_plain_form(case, cap, slope, window, sink, span):
    x = make(case)
    opt = options(case, cap, slope, window, sink, span)
    got = run(case, x[0], x, opt)
    check(got, pref.scored_reference(*x[:5], case[8], **opt), case, opt)
