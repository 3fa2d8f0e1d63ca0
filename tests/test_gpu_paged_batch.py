"""StitchedBatch on a pair of models whose caches are in pages: each sequence's run is that of the oracle, pages are handed on from one batch to the next."""
import math

import pytest
import torch

import workloads as W
from oracle import decoder, stitch

pytestmark = pytest.mark.gpu


def test_a_batch_in_pages_matches_the_single_sequence_runs():
    import paper_2507_17307_amd as P
    from paper_2507_17307_amd.stitch import StitchedBatch
    wl, lens, n_new, page = W.WORKLOADS["cfg1_tiny_pair"], [20, 32, 7, 45], 24, 16
    max_ctx = max(lens) + n_new + 3
    weights = [W.make_weights(wl.slm, wl.seed, 0), W.make_weights(wl.llm, wl.seed, 1)]
    prompts = [W.make_prompt(wl, seq=b, length=n).tolist() for b, n in enumerate(lens)]
    scales = [W.logit_scale(wl, 0, max_ctx + 1, seq=b) for b in range(4)]
    mk = lambda: [decoder.OracleModel(w, max_ctx + 1) for w in weights]  # noqa: E731
    hs = [t.h_norm for p, s in zip(prompts, scales) for t in stitch.generate(p, stitch.decoder_forward(mk(), lambda i, s=s: float(s[i])), 2.0, n_new).trace]
    tau = W.pick_tau(hs, 60.0, 4e-3 / math.log(wl.slm.vocab))
    want = [stitch.generate(p, stitch.decoder_forward(mk(), lambda i, s=s: float(s[i])), tau, n_new) for p, s in zip(prompts, scales)]
    need = [-(-(len(p) + n_new) // page) for p in prompts]
    gpu = [P.PagedModel(w.to("cuda"), max_ctx=max_ctx + 1, n_pages=sum(need), page_size=page, max_seqs=4, max_rows=64) for w in weights]
    batch = StitchedBatch(gpu[0], gpu[1], max_ctx, scales)
    for order in ((0, 1, 2, 3), (2, 0, 3, 1)):                                 # the second time other pages for each
        for m in gpu:
            for b in order:
                m.reserve(b, len(prompts[b]) + n_new)
        torch.cuda.synchronize()
        runs = batch.generate(prompts, tau, n_new)
        for run, ref in zip(runs, want):
            assert run.output == ref.output
            assert [(t.model, t.pos0, t.n_rows, t.accept) for t in run.trace] == [(t.model, t.pos0, len(t.span), t.accept) for t in ref.trace]
        for m in gpu:
            for b in reversed(order):
                m.release(b)
    for m in gpu:
        m.close()
