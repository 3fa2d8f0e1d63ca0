"""A beam search on a model that has other sequences too: the slots beyond the search's rows keep what they have."""
import pytest
import torch

import workloads as W
from test_gpu_beam_search import tokens


@pytest.mark.gpu
def test_slots_beyond_the_search_keep_their_pages():
    """One slot has a sequence from before the hand-over, another gets one from the pool later; both go on as if there had been no search."""
    import paper_2507_17307_amd as P
    w = W.make_weights(W.TINY_S, seed=5, role=0).to("cuda")
    lines = [tokens(W.TINY_S, 40, 80), tokens(W.TINY_S, 40, 81)]
    alone = P.Model(w, max_ctx=64, max_seqs=2, max_rows=32)
    want = [alone.forward_span(line[:30], 0, 0.8, P.RS_LLM, slot=s)[0] for s, line in enumerate(lines)] + \
           [alone.forward_span(line[30:31], 30, 0.8, P.RS_LLM, slot=s)[0] for s, line in enumerate(lines)]
    model = P.PagedModel(w, max_ctx=64, n_pages=24, page_size=16, max_seqs=7, max_rows=32)
    model.reserve(5, 40)
    got = [model.forward_span(lines[0][:30], 0, 0.8, P.RS_LLM, slot=5)[0]]
    search = P.BeamSearch(model, 1, 4, logit_scale=6.0)
    ints = [torch.tensor([v], dtype=torch.int32, device="cuda") for v in (6, 40)]
    P.rs_pages_reserve(search.pool, 1, ints[0], None, ints[1], search.pool_scratch)
    got.append(model.forward_span(lines[1][:30], 0, 0.8, P.RS_LLM, slot=6)[0])
    torch.cuda.synchronize()
    table, pages = model.page_table[5:].clone(), [model.kv_view(which, slot).clone() for slot in (5, 6) for which in "kv"]
    prompt = tokens(W.TINY_S, 13, 70)
    first = search.generate([prompt], 20)
    assert search.generate([prompt], 20) == first
    assert torch.equal(model.page_table[5:], table)
    assert bool((search.pool.page_ref[table[table >= 0].long()] == 1).all())
    for before, (slot, which) in zip(pages, [(s, which) for s in (5, 6) for which in "kv"]):
        assert torch.equal(model.kv_view(which, slot), before)
    held = model.page_table[model.page_table >= 0].long()
    assert torch.equal(search.pool.page_ref, torch.bincount(held, minlength=24).to(torch.int32))
    got += [model.forward_span(line[30:31], 30, 0.8, P.RS_LLM, slot=s)[0] for s, line in zip((5, 6), lines)]
    torch.cuda.synchronize()
    assert [g.token for g in got] == [x.token for x in want] and all(g.flags == x.flags for g, x in zip(got, want))
    # the same search with all of the pool to itself
    own = P.PagedModel(w, max_ctx=64, n_pages=24, page_size=16, max_seqs=4, max_rows=32)
    assert P.BeamSearch(own, 1, 4, logit_scale=6.0).generate([prompt], 20) == first
    model.close(), own.close(), alone.close()


@pytest.mark.gpu
def test_a_smaller_search_has_the_pages_of_a_larger_one():
    """Sixteen pages: eight beams of 18 tokens leave 7 in the slots beyond the first four, which four beams of 50 tokens, that need 14, have again; of a
    search made before the larger one and of one made after it."""
    import paper_2507_17307_amd as P
    w = W.make_weights(W.TINY_S, seed=5, role=0).to("cuda")
    prompt, other = tokens(W.TINY_S, 13, 70), tokens(W.TINY_S, 13, 73)
    calls = {1: ([prompt], 50), 2: ([prompt, other], 18)}

    def model_of(n_pages):
        return P.PagedModel(w, max_ctx=64, n_pages=n_pages, page_size=16, max_seqs=8, max_rows=8)
    want = {}
    for n, call in calls.items():
        model = model_of(40)
        want[n] = P.BeamSearch(model, n, 4, logit_scale=6.0).generate(*call)
        model.close()
    model = model_of(16)
    early, large, late = (P.BeamSearch(model, n, 4, logit_scale=6.0) for n in (1, 2, 1))
    for search in (large, late, large, early):
        assert search.generate(*calls[search.n_prompts]) == want[search.n_prompts]
        held = model.page_table[model.page_table >= 0].long()
        assert torch.equal(large.pool.page_ref, torch.bincount(held, minlength=16).to(torch.int32))
    model.close()
