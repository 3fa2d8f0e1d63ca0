"""rs_paged_attention over many tiles: sums that are relative to the running maximum stay so while it does not change."""
import numpy as np
import pytest
import torch

import paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,group,seqs,rows", [(torch.float32, 1, 1024, 1), (torch.float32, 16, 600, 1), (torch.float32, 8, 300, 4), (torch.float32, 16, 1, 9), (torch.bfloat16, 16, 600, 1),
                                                   (torch.bfloat16, 4, 1, 30), (torch.bfloat16, 2, 20, 1)])
def test_equal_scores_weigh_the_same_however_many_tiles_there_are(dtype, group, seqs, rows):
    """16000 positions of one score, about 4000: lse is the score and the logarithm of their number, out the mean of V, which is 0 in the first half of the positions and 1 in
    the second.  The sequences read one slot, so that a run has whole items.

    How far: every probability is the same number, so that sums of n terms are off by at most n roundings, relative to the sum, in out three times (the planes of p; V is 0 or
    1), and once more for the sum that it is divided by; the score and the factor log2 e are rounded, and the score's place in the exponent."""
    import paper_2507_17307_amd as P
    length, page, hd = 16000, 1024, 32
    n_pages = -(-length // page)
    k = torch.ones(n_pages, 1, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(n_pages, 1, hd, page, dtype=torch.bfloat16, device="cuda")
    at = torch.arange(n_pages * page, device="cuda").view(n_pages, 1, 1, page)
    v[:] = (at >= length // 2).to(torch.bfloat16)
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    cache = P.PagedCache(k, v, table)
    # a q (a whole number, exact in bf16) whose score's place in the exponent is far from a float: that is where a sum can lose its reference
    c = np.float32(0.5) * np.float32(1.44269504088896341)
    best = max((x for x in np.arange(248, 256, 1 / 16) if float(torch.tensor(x).bfloat16()) == x), key=lambda x: abs(float(np.float32(32 * x)) * float(c) - float(np.float32(32 * x) * c)))
    n = seqs * rows
    q = torch.full((n, group, hd), best, dtype=dtype, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n, group, device="cuda")
    slot = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    off = torch.arange(0, n + 1, rows, dtype=torch.int32, device="cuda")
    pos = torch.full((seqs,), length - rows, dtype=torch.int32, device="cuda")
    scratch = torch.empty(P.rs_paged_attention_scratch_bytes(cache, seqs, n, group), dtype=torch.uint8, device="cuda")
    P.rs_paged_attention(cache, seqs, n, slot, off, pos, q, 0.5, 0, out, lse, scratch)
    seen = (length - rows + 1 + torch.arange(rows, dtype=torch.float64)).repeat(seqs)[:, None]
    s = 32 * best * 0.5
    e_sum = length * paged.F32
    off_lse = (lse.cpu().double() - (s + seen.log())).abs()
    assert float(off_lse.max()) <= 4 * paged.F32 * s + e_sum + 2.0 ** -20
    want = (seen - length // 2) / seen
    paged.close(out.cpu(), want[..., None].expand(out.shape), 4 * e_sum * want[..., None].expand(out.shape))
