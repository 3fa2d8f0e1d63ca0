"""A sequence of a paged model that misses a page: nothing of it is computed or written, and once the page is there its tokens can be fed again."""
import pytest
import torch

import workloads as W
from oracle import decoder
from parity import check_invocation
from test_gpu_paged_model import tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("p0,rows,gone", [(0, 17, 1), (0, 40, 1), (15, 2, 1), (14, 4, 1), (0, 40, 0), (30, 1, 0), (33, 1, 1), (31, 3, 0), (20, 9, 0), (40, 20, 1)])
@pytest.mark.parametrize("entry", [-1, 10 ** 6])
def test_a_sequence_that_misses_a_page_leaves_the_cache_as_it_is(p0, rows, gone, entry):
    """The page of the last rows, of rows in the middle, of positions before the call's; one row, few (side by side) and many (matrix cores), another sequence beside them."""
    import paper_2507_17307_amd as P
    shape = W.TINY_S
    w = W.make_weights(shape, seed=11, role=0)
    gpu = P.PagedModel(w.to("cuda"), max_ctx=64, n_pages=8, page_size=16, max_seqs=2, max_rows=64)
    refs = [decoder.OracleModel(w, 64) for _ in range(2)]
    toks = [tokens(shape, 64, 80), tokens(shape, 64, 81)]
    gpu.reserve(0, p0 + rows)
    gpu.reserve(1, 20)
    if p0:
        refs[0].forward(toks[0][:p0], 0)
        gpu.forward_span(toks[0][:p0], 0, 0.8, P.RS_SLM, slot=0)
    held = gpu.page_table[0, gone].item()
    gpu.page_table[0, gone] = entry
    before = gpu.kv_view("k", 0).clone(), gpu.kv_view("v", 0).clone()
    want = [r.forward(t[p:p + n], p)["logits"] for r, t, p, n in zip(refs, toks, (p0, 0), (rows, 2))]

    def call(slots, spans, pos):
        if all(len(s) == 1 for s in spans):
            return gpu.decode_step([s[0] for s in spans], pos, 0.8, P.RS_SLM, slots=slots, want_logits=True)
        return gpu.catchup_prefill(spans, pos, 0.8, P.RS_SLM, slots=slots, want_logits=True)
    got, logits = call([0, 1], [toks[0][p0:p0 + rows], toks[1][:2 if rows > 1 else 1]], [p0, 0])
    assert got[0].flags & P.FLAG_BADARG
    if rows > 1:
        check_invocation(got[1], logits[1], want[1], 0.8, P.RS_SLM)
    assert torch.equal(gpu.kv_view("k", 0), before[0]) and torch.equal(gpu.kv_view("v", 0), before[1])
    gpu.page_table[0, gone] = held
    got, logits = call([0], [toks[0][p0:p0 + rows]], [p0])
    check_invocation(got[0], logits[0], want[0], 0.8, P.RS_SLM)
    gpu.close()
