"""Which pages a beam search takes: those of the beams that run, beams that ended or are not there hold none."""
import dataclasses

import pytest
import torch

import beam
import workloads as W
from test_gpu_beam_search import oracle_search, tokens

pytestmark = pytest.mark.gpu

PAGE = 16


def model_of(w, n_pages, rows):
    import paper_2507_17307_amd as P
    return P.PagedModel(w, max_ctx=64, n_pages=n_pages, page_size=PAGE, max_seqs=rows, max_rows=rows)


def traced(model, *args, **more):
    """A search that keeps the steps' parents and tokens."""
    import paper_2507_17307_amd as P

    class Traced(P.BeamSearch):
        def _read(self, parents, tokens, scores):
            self.trace = parents, tokens
            return super()._read(parents, tokens, scores)
    return Traced(model, *args, **more)


def suffices(n_pages, prompts, n_beams, eos, trace, all_rows):
    """Whether a search with these steps gets by with so many pages: those of its running beams, or (all_rows) of every row."""
    rows = len(prompts) * n_beams
    pool, slot = beam.PoolModel(rows, 64 // PAGE, n_pages, PAGE), list(range(rows))
    pos = [len(prompts[r // n_beams]) if r % n_beams == 0 else 0 for r in slot]
    if any(pool.reserve(slot, [0] * rows, pos)):
        return False
    for step, (parent, token) in enumerate(zip(*trace)):
        if step:
            end = [p + (all_rows or a) for p, a in zip(pos, runs)]
            if any(pool.reserve(slot, pos, end)):
                return False
            pos = end
        runs = [t >= 0 and t != eos for t in token]
        flags, pos = pool.fork(n_beams, slot, [p if all_rows or a else -1 for p, a in zip(parent, runs)], pos)
        if any(flags):
            return False
    return True


def searched_in_the_pages_of_running_beams(w, prompts, n_beams, n_tokens, eos, scale, check_every):
    """The results in plenty of pages; a pool that is just large enough for the beams that run gives the same."""
    rows = len(prompts) * n_beams
    plenty = model_of(w, rows * 4 + 8, rows)
    search = traced(plenty, len(prompts), n_beams, eos, logit_scale=scale)
    want = search.generate(prompts, n_tokens, check_every)
    trace = search.trace
    least = next(n for n in range(1, rows * 4 + 8) if suffices(n, prompts, n_beams, eos, trace, False))
    assert not suffices(least, prompts, n_beams, eos, trace, True)
    tight = model_of(w, least, rows)
    search = traced(tight, len(prompts), n_beams, eos, logit_scale=scale)
    for again in range(2):
        assert search.generate(prompts, n_tokens, check_every) == want
        assert search.trace == trace
    held = tight.page_table[tight.page_table >= 0].long()
    assert torch.equal(search.pool.page_ref, torch.bincount(held, minlength=least).to(torch.int32))
    plenty.close(), tight.close()
    return want, trace


@pytest.mark.parametrize("check_every", [0, 16])
@pytest.mark.parametrize("n_beams, n_tokens, eos, lengths", [(4, 48, 438, [1, 5, 6, 48]), (1, 30, 340, [1])])
def test_ended_beams_hold_no_pages(n_beams, n_tokens, eos, lengths, check_every):
    """Of four beams three end within six tokens and one goes on; a single one ends at once, and the steps that follow (unless the host looks) have no row that runs."""
    w = W.make_weights(W.TINY_S, seed=5, role=0)
    prompt, scale = tokens(W.TINY_S, 13, 70), 4.0
    want, gap = oracle_search(w, prompt, n_beams, n_tokens, eos, 0.0, scale)
    assert gap > 1e-3 and [len(line) for line, _ in want] == lengths
    got, _ = searched_in_the_pages_of_running_beams(w.to("cuda"), [prompt], n_beams, n_tokens, eos, scale, check_every)
    assert [b.tokens for b in got[0]] == [line for line, _ in want]
    assert all(abs(b.score - s) <= 1e-3 * n_tokens for b, (_, s) in zip(got[0], want))
    assert [b.ended for b in got[0]] == [line[-1] == eos for line, _ in want]


def test_one_prompts_beams_end_beside_others_that_run():
    w = W.make_weights(W.TINY_S, seed=5, role=0)
    prompts = [tokens(W.TINY_S, 13, 70), tokens(W.TINY_S, 31, 75)]
    got, _ = searched_in_the_pages_of_running_beams(w.to("cuda"), prompts, 4, 30, 438, 4.0, 16)
    assert [len(b.tokens) for b in got[0]] == [1, 5, 6, 30] and [len(b.tokens) for b in got[1]] == [30] * 4


def test_absent_beams_hold_no_pages():
    """Five tokens for eight beams: three of them are not there before the second step.  That one fills the prompts' pages, which the beams then share, so
    that the most pages are held between the two."""
    shape = dataclasses.replace(W.TINY_S, name="tiny_v", vocab=5)
    w = W.make_weights(shape, seed=5, role=0).to("cuda")
    prompts = [[1, 4, 2, 0, 3] * 3, [2, 2, 0, 4, 1] * 3]
    rows = 16
    got, trace = searched_in_the_pages_of_running_beams(w, prompts, 8, 2, -1, 3.0, 0)
    assert [sum(t < 0 for t in tokens) for tokens in trace[1]] == [6, 0] and [len(g) for g in got] == [8, 8]
    # behind a search of one token the rows that are not there hold nothing
    model = model_of(w, 64, rows)
    search = traced(model, 2, 8, logit_scale=3.0)
    assert [len(g) for g in search.generate(prompts, 1)] == [5, 5]
    gone = torch.tensor([t < 0 for t in search.trace[1][0]]).cuda()
    assert int(gone.sum()) == 6 and bool((model.page_table[gone] == -1).all())
    model.close()
