"""rs_paged_attention: an infinity or a NaN in V reaches every row that sees it, whatever the scores of the positions behind it are."""
import math

import pytest
import torch

import paged
from test_gpu_paged_attention import call, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("spans,pos0,window", [([1], [200], 0), ([1] * 40, [200 + i for i in range(40)], 0), ([3, 2], [200, 700], 0), ([60], [190], 0), ([300], [0], 0),
                                               ([20] * 40, [180 + i for i in range(40)], 0), ([90], [150], 120)])
def test_a_later_score_that_is_much_higher_does_not_turn_an_infinity_into_a_nan(spans, pos0, window, bad, dtype):
    """One position's score is 160 above the others': beside it they are 0 in 32 bits, and an infinity of theirs is still an infinity of the sum."""
    pg = paged.Pages(spans, pos0, 2, 64, 16, seed=60)
    for b in range(len(spans)):
        page = [int(p) for p in pg.table[pg.slot[b]]]
        pg.k[page[160 // 16], :, 160 % 16] = 20.0
        for at, chan in ((95, 3), (130, 40), (170, 3)):
            pg.v[page[at // 16], at % 2, chan, at % 16] = bad
    pg.gpu()
    q = (1.0 + 0.1 * torch.randn(pg.rows, 8, 64, generator=pg.gen)).to(dtype)
    out, lse = call(pg, q, 0.125, window)
    check(pg, q, 0.125, window, out, lse)
