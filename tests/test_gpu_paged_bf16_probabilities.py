"""rs_paged_attention on bf16 rows: the bits of the probabilities."""
import pytest
import torch

import paged
from test_gpu_paged_attention import call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spans,pos0,nq,nkv", [([1], [700], 28, 4), ([1] * 70, [(29 * i) % 900 for i in range(70)], 28, 4), ([1] * 9, [100 * i for i in range(9)], 64, 4),
                                               ([2, 1, 3, 1] * 12, [(53 * i) % 600 for i in range(48)], 16, 2), ([7, 5], [300, 900], 14, 2), ([20] * 9, [(77 * i) % 800 for i in range(9)], 16, 4),
                                               ([24] * 3 + [1] * 30, [(31 * i) % 300 for i in range(33)], 32, 8), ([32] * 9, [(77 * i) % 800 for i in range(9)], 16, 4)])
def test_the_probabilities_of_bf16_rows_have_more_bits_than_the_output(spans, pos0, nq, nkv):
    """Single tokens and short spans (rows times query heads of a KV head up to 128), however many sequences they are called with: the error is that of
    fp32 rows, 2^-16 of a term (two roundings to bf16) and the output's rounding."""
    pg = paged.Pages(spans, pos0, nkv, 128, 32, seed=61).gpu()
    q = (0.5 * torch.randn(pg.rows, nq, 128, generator=pg.gen)).to(torch.bfloat16)
    out, lse = call(pg, q, 128 ** -0.5)
    want, z, eo, ez = paged.attention(pg, q.float(), 128 ** -0.5)                       # (as fp32 rows: the bound without a rounding of p)
    mean_v = torch.zeros_like(want)
    r = 0
    for b, (m, p0) in enumerate(zip(spans, pos0)):                                     # sum p |v| <= max |v|
        mean_v[r:r + m] = pg.held(b)[1].abs().double().amax(0).repeat_interleave(nq // nkv, 0)
        r += m
    paged.close(out, want, eo + 2.0 ** -16 * mean_v)
    paged.close(lse, z, ez)
