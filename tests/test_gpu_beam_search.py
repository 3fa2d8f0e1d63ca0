"""Beam search on a model in pages (selection, forks, reserved pages and decode steps together) against the oracle, beam by beam, and against the
same model by slots fed with what came out."""
import math

import pytest
import torch

import workloads as W
from oracle import decoder
from workloads.recipes import misc_normal


def tokens(shape, n, seed):
    return (torch.abs(misc_normal(seed, 0, n)) * 1e4).long().remainder(shape.vocab).tolist()


def oracle_search(w, prompt, n_beams, n_tokens, eos, alpha, scale):
    """([(tokens, score)] in order, the least gap of a rank that decided something) in 64 bits, every beam from its first token on."""
    model = decoder.OracleModel(w, len(prompt) + n_tokens)
    beams, gap = [([], 0.0)], math.inf
    for _ in range(n_tokens):
        found = []
        for b, (toks, score) in enumerate(beams):
            if eos >= 0 and toks and toks[-1] == eos:
                found.append((score / max(toks.index(eos) + 1, 1) ** alpha, b, eos, score))
                continue
            x = model.forward(prompt + toks, 0, logit_scale=scale)["logits"]
            lp = torch.log_softmax(x, 0)
            best = torch.topk(lp, n_beams + 1)
            found += [(float(score + l) / (len(toks) + 1) ** alpha, b, int(t), score + float(l)) for l, t in zip(best.values, best.indices)]
        found.sort(key=lambda f: (-f[0], f[1]))
        gap = min([gap] + [a[0] - b[0] for a, b in zip(found[:n_beams], found[1:n_beams + 1])])
        beams = [(beams[b][0] + [t], s) for _, b, t, s in found[:n_beams]]
    cut = [toks[:toks.index(eos) + 1] if eos >= 0 and eos in toks else toks for toks, _ in beams]
    return [(c, s) for c, (_, s) in zip(cut, beams)], gap


# shape, page size, prompts, beams, tokens, eos, length penalty, logit scale
CASES = [(W.TINY_S, 16, (0, 2, 3), 4, 20, -1, 0.0, 6.0), (W.TINY_L, 16, (0, 3, 6), 5, 19, -1, 0.0, 8.0), (W.TINY_S, 32, (2,), 8, 10, 765, 0.7, 5.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape, page, which, n_beams, n_tokens, eos, alpha, scale", CASES)
def test_beams_are_the_oracles(shape, page, which, n_beams, n_tokens, eos, alpha, scale):
    import paper_2507_17307_amd as P
    w = W.make_weights(shape, seed=5, role=0)
    n_prompts, prompts = len(which), [tokens(shape, 13 + 9 * (i % 3), 70 + i) for i in which]
    want = [oracle_search(w, p, n_beams, n_tokens, eos, alpha, scale) for p in prompts]
    # logits of the two differ by less than 1e-3 (scaled, of values of some tens); what lies nearer is left out by the choice of seeds
    assert min(gap for _, gap in want) > 1e-3
    gpu = P.PagedModel(w.to("cuda"), max_ctx=96, n_pages=n_prompts * n_beams * 4 + 8, page_size=page, max_seqs=n_prompts * n_beams, max_rows=n_prompts * n_beams)
    search = P.BeamSearch(gpu, n_prompts, n_beams, eos, alpha, scale)
    for again in range(2):                                                    # the second time from slots that hold something, replayed
        got = search.generate(prompts, n_tokens)
        for g in range(n_prompts):
            assert [b.tokens for b in got[g]] == [t for t, _ in want[g][0]], f"prompt {g}"
            assert all(abs(b.score - s) <= 1e-3 * n_tokens for b, (_, s) in zip(got[g], want[g][0]))
            assert [b.ended for b in got[g]] == [eos >= 0 and t[-1] == eos for t, _ in want[g][0]]
    # every page is counted as often as the table names it
    held = gpu.page_table[gpu.page_table >= 0].long()
    assert torch.equal(search.pool.page_ref, torch.bincount(held, minlength=gpu.n_pages).to(torch.int32))
    gpu.close()


@pytest.mark.gpu
def test_scores_are_those_of_the_sequences_fed_from_the_start():
    """64 beams of long replies over small pages: what each beam scored step by step, from shared and copied pages, is what its tokens get in one span each."""
    import paper_2507_17307_amd as P
    shape = W.TINY_L
    w = W.make_weights(shape, seed=9, role=0).to("cuda")
    prompts = [tokens(shape, n, 90 + n) for n in (5, 16, 40, 31)]
    paged = P.PagedModel(w, max_ctx=160, n_pages=500, page_size=16, max_seqs=64, max_rows=64)
    got = P.BeamSearch(paged, 4, 16, logit_scale=7.0).generate(prompts, 70)
    plain = P.Model(w, max_ctx=160, max_seqs=1, max_rows=64)
    for prompt, beams in zip(prompts, got):
        assert len(beams) == 16 and len({tuple(b.tokens) for b in beams}) == 16
        assert all(a.score >= b.score for a, b in zip(beams, beams[1:]))
        for beam in (beams[0], beams[7], beams[15]):
            score, line = 0.0, prompt + beam.tokens
            for at in range(len(prompt), len(line)):
                _, logits = plain.forward_span(line[at - 1:at], at - 1, 0.5, P.RS_LLM, want_logits=True) if at > len(prompt) else \
                    plain.forward_span(prompt, 0, 0.5, P.RS_LLM, want_logits=True)
                score += float(torch.log_softmax(logits[0].double() * 7.0, 0)[line[at]])
            assert abs(beam.score - score) <= 2e-3 * len(beam.tokens), (beam.score, score)
    paged.close(), plain.close()


@pytest.mark.gpu
def test_too_few_pages_are_told_and_pages_belong_to_the_pool():
    import paper_2507_17307_amd as P
    w = W.make_weights(W.TINY_S, seed=5, role=0).to("cuda")
    model = P.PagedModel(w, max_ctx=64, n_pages=5, page_size=16, max_seqs=4, max_rows=4)
    for more in (dict(eos=-2), dict(eos=W.TINY_S.vocab), dict(length_penalty=-1.0), dict(length_penalty=31.0), dict(logit_scale=0.0)):
        with pytest.raises(ValueError):
            P.BeamSearch(model, 1, 4, **more)
    model.reserve(2, 20)                                                      # (the pages are still the model's)
    search = P.BeamSearch(model, 1, 4, logit_scale=6.0)
    assert search.pool.page_ref.tolist() == [1, 1, 0, 0, 0]
    with pytest.raises(P.RsError, match="pages"):
        search.generate([tokens(W.TINY_S, 10, 1)], 30)
    assert [len(b.tokens) for b in search.generate([tokens(W.TINY_S, 10, 1)], 5)[0]] == [5] * 4
    for call in (lambda: model.reserve(0, 16), lambda: model.release(2)):
        with pytest.raises(P.RsError, match="pool"):
            call()
    for args in ((2, 4), (1, 5), (0, 4)):
        with pytest.raises(ValueError):
            P.BeamSearch(model, *args)
    with pytest.raises(ValueError):
        search.generate([[1] * 40], 30)
    for prompt in ([], [1, W.TINY_S.vocab], [-1]):
        with pytest.raises(ValueError):
            search.generate([prompt], 3)
    model.close()
