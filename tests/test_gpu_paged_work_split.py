"""rs_paged_attention's split of the work where it has many blocks or many items: long spans with many query heads a KV head, runs of more than 32 items, and the pieces of
a cut item found again when its sums hold a NaN."""
import math

import pytest
import torch

import paged
from test_gpu_paged_attention import call, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [None, math.nan])
@pytest.mark.parametrize("spans,pos0,window", [([1300], [5], 0), ([1300, 3], [70, 200], 90), ([2] + [530] + [1] * 20, [i * 7 for i in range(22)], 0),
                                               ([300] + [1] * 500, [40] + [i % 60 for i in range(500)], 0)])
def test_spans_of_more_than_64_blocks(spans, pos0, window, bad, dtype):
    """16 query heads a KV head: a block has 8, 2 or 1 rows, so that these spans have up to 165 of them."""
    pg = paged.Pages(spans, pos0, 1, 32, 16, seed=70, fill=math.inf)
    if bad is not None:
        long = max(range(len(spans)), key=lambda b: spans[b])
        at = pos0[long] + spans[long] * 3 // 4
        pg.v[pg.table[pg.slot[long], at // 16], 0, 9, at % 16] = bad
    pg.gpu()
    q = torch.randn(pg.rows, 16, 32, generator=pg.gen).to(dtype)
    out, lse = call(pg, q, 0.2, window)
    check(pg, q, 0.2, window, out, lse)


@pytest.mark.parametrize("dtype,group,rows,n_kv", [(torch.float32, 1, 1, 64), (torch.float32, 12, 2, 64), (torch.float32, 12, 4, 16), (torch.bfloat16, 1, 1, 32), (torch.bfloat16, 16, 3, 24)])
def test_runs_of_more_than_32_items(dtype, group, rows, n_kv):
    """1024 sequences of one tile: every run has 48 to 64 whole items, and infinities and NaN lie in every ninth sequence's V, in KV heads that differ from one to the next."""
    n = 1024
    pg = paged.Pages([rows] * n, [(5 * i) % 13 for i in range(n)], n_kv, 32, 16, seed=71, fill=math.inf, spare_pages=0)
    for b in range(0, n, 9):
        p = pg.pos0[b] // 2
        for h in range(b % 5, n_kv, 7):
            pg.v[pg.table[pg.slot[b], p // 16], h, (b + h) % 32, p % 16] = (math.inf, math.nan, -math.inf)[(b + h) % 3]
    pg.gpu()
    q = torch.randn(pg.rows, group * n_kv, 32, generator=pg.gen).to(dtype)
    out, lse = call(pg, q, 0.2)
    check(pg, q, 0.2, 0, out, lse)
