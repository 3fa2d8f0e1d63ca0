"""Models whose cache is in pages (rs_create_model_paged) against the oracle: every path a call can take, pages in any order, pages that are missing,
pages handed on, the host driver's stitched loop on a pair of them."""
import math

import pytest
import torch

import workloads as W
from oracle import decoder
from parity import check_invocation
from test_gpu_model import pair_run
from workloads.recipes import misc_normal

pytestmark = pytest.mark.gpu

WIDE = W.ModelShape("wide", 2, 256, 6, 2, 64, 384, 1024, False)               # three query heads a KV head, 64 channels
BIG = W.ModelShape("big", 2, 2176, 17, 17, 128, 512, 1024, False)             # a query head each, too wide for four rows side by side


def tokens(shape, n, seed):
    return (torch.abs(misc_normal(seed, 0, n)) * 1e4).long().remainder(shape.vocab).tolist()


@pytest.mark.parametrize("shape,page", [(W.TINY_S, 16), (W.TINY_L, 64), (WIDE, 32), (BIG, 16)])
def test_spans_and_steps_match_the_oracle(shape, page):
    """Three sequences in one pool: prompts in spans of every size class (one row, two, four, a matrix-core call of up to 16 and of more rows), then steps."""
    import paper_2507_17307_amd as P
    w = W.make_weights(shape, seed=5, role=0)
    gpu = P.PagedModel(w.to("cuda"), max_ctx=200, n_pages=-(-170 // page) + 2 * (-(-60 // page)), page_size=page, max_seqs=3, max_rows=64)
    refs = [decoder.OracleModel(w, 200) for _ in range(3)]
    toks = [tokens(shape, n, 40 + i) for i, n in enumerate((170, 60, 60))]
    at = [0, 0, 0]
    # rows that the three sequences bring, call by call
    calls = [(33, 5, 0), (0, 0, 1), (60, 0, 2), (2, 0, 0), (1, 1, 1), (4, 7, 2), (0, 1, 1), (17, 3, 3), (0, 2, 0), (1, 0, 0), (30, 31, 3), (1, 1, 1)]
    for k, rows in enumerate(calls):
        seqs = [b for b in range(3) if rows[b]]
        for b in seqs:
            gpu.reserve(b, at[b] + rows[b])
        spans, pos = [toks[b][at[b]:at[b] + rows[b]] for b in seqs], [at[b] for b in seqs]
        scales = [0.7 + 0.4 * b + 0.1 * k for b in seqs]
        if max(rows) == 1:
            got, logits = gpu.decode_step([s[0] for s in spans], pos, 0.8, P.RS_SLM, scales, seqs, want_logits=True)
        else:
            got, logits = gpu.catchup_prefill(spans, pos, 0.8, P.RS_SLM, scales, seqs, want_logits=True)
        for i, b in enumerate(seqs):
            want = refs[b].forward(spans[i], pos[i], logit_scale=scales[i])["logits"]
            check_invocation(got[i], logits[i], want, 0.8, P.RS_SLM, where=f"call {k} sequence {b}")
            at[b] += rows[b]
    gpu.close()


@pytest.mark.parametrize("page", [16, 1024])
def test_the_rows_written_are_those_of_a_model_by_slots(page):
    """First layer's K and V bit for bit (the same products and rotations), at every row count class; the later layers' within what one bf16 step makes of them."""
    import paper_2507_17307_amd as P
    shape = W.TINY_L
    w = W.make_weights(shape, seed=6, role=0).to("cuda")
    slots = P.Model(w, max_ctx=128, max_seqs=2, max_rows=128)
    pages = P.PagedModel(w, max_ctx=128, n_pages=2 * max(1, 128 // page), page_size=page, max_seqs=2, max_rows=128)
    toks = tokens(shape, 128, 50)
    for b in (1, 0):
        pages.reserve(b, 100)
    p = 0
    for n in (1, 2, 4, 16, 40, 37):
        for m in (slots, pages):
            m.catchup_prefill([toks[p:p + n], toks[p + 1:p + 1 + n]], [p, p], 0.5, P.RS_SLM, slots=[0, 1])
        p += n
    for which in ("k", "v"):
        for b in (0, 1):
            have, want = pages.kv_view(which, b)[:, :, :100], slots.kv_view(which)[:, b, :, :100]
            assert torch.equal(have[0], want[0])
            assert float((have.float() - want.float()).norm() / want.float().norm()) <= 2.0 ** -8
    for m in (slots, pages):
        m.close()


def test_a_missing_page_is_flagged_and_the_others_go_on():
    import paper_2507_17307_amd as P
    shape = W.TINY_S
    w = W.make_weights(shape, seed=7, role=0)
    gpu, ref = P.PagedModel(w.to("cuda"), max_ctx=64, n_pages=6, page_size=16, max_seqs=3), decoder.OracleModel(w, 64)
    toks = tokens(shape, 40, 60)
    gpu.reserve(0, 33)
    gpu.reserve(1, 16)
    gpu.reserve(2, 8)
    gpu.page_table[2, 0] = 10 ** 6
    want = ref.forward(toks[:30], 0)["logits"]
    got, logits = gpu.catchup_prefill([toks[:30], toks[:17], toks[:3]], [0, 0, 0], 0.8, P.RS_SLM, want_logits=True)
    check_invocation(got[0], logits[0], want, 0.8, P.RS_SLM)
    assert got[1].flags & P.FLAG_BADARG and got[2].flags & P.FLAG_BADARG
    # a sequence whose last row has its page and an earlier one has not
    gpu.page_table[0, 0] = -1
    got = gpu.decode_step([toks[30]], [30], 0.8, P.RS_SLM, slots=[0])
    assert got[0].flags & P.FLAG_BADARG
    with pytest.raises(P.RsError):
        gpu.reserve(2, 64)
    with pytest.raises(P.RsError):
        gpu.reserve(0, 80)
    gpu.close()


def test_pages_are_handed_on():
    """A slot's pages go to another sequence in another order; what the first one left there does not show."""
    import paper_2507_17307_amd as P
    shape = W.TINY_S
    w = W.make_weights(shape, seed=8, role=0)
    gpu = P.PagedModel(w.to("cuda"), max_ctx=64, n_pages=4, page_size=16, max_seqs=2)
    a, b = tokens(shape, 60, 70), tokens(shape, 60, 71)
    gpu.reserve(0, 64)
    gpu.forward_span(a, 0, 0.8, P.RS_SLM)
    gpu.pages_v.mul_(float("nan"))                                          # the worst that can be left behind
    gpu.release(0)
    ref = decoder.OracleModel(w, 64)
    at = 0
    for n in (20, 1, 30):
        gpu.reserve(1, at + n)
        want = ref.forward(b[at:at + n], at, logit_scale=2.0)["logits"]
        got, logits = gpu.forward_span(b[at:at + n], at, 0.8, P.RS_SLM, 2.0, slot=1, want_logits=True)
        check_invocation(got[0], logits[0], want, 0.8, P.RS_SLM)
        at += n
    gpu.close()


def test_the_stitched_loop_on_a_pair_in_pages_is_the_oracle_run():
    import paper_2507_17307_amd as P
    from paper_2507_17307_amd.stitch import StitchedPair
    wl = W.WORKLOADS["cfg1_tiny_pair"]
    weights, _, res, _, tau, scales = pair_run(wl)
    pages = -(-(wl.max_ctx + 8) // 16)
    gpu = [P.PagedModel(w.to("cuda"), max_ctx=wl.max_ctx + 1, n_pages=pages, page_size=16, max_rows=64) for w in weights]
    for m in gpu:
        m.reserve(0, wl.max_ctx + 1)
    pair = StitchedPair(gpu[0], gpu[1], wl.max_ctx, scales)
    prompt = W.make_prompt(wl).tolist()
    for _ in range(2):                                                        # the second run replays the first one's graphs
        run = pair.generate(prompt, tau, wl.n_decode)
        assert run.output == res.output
        assert [(t.model, t.pos0, t.n_rows, t.accept) for t in run.trace] == [(t.model, t.pos0, len(t.span), t.accept) for t in res.trace]
        assert max(abs(a.h_norm - b.h_norm) for a, b in zip(run.trace, res.trace)) <= 1e-3 / math.log(1024)
    with pytest.raises(P.RsError) as e:
        pair.generate_on_device(prompt, tau, wl.n_decode)
    assert e.value.status == -4 and "slots" in str(e.value)


def test_models_that_do_not_fit_their_pages_are_refused():
    import ctypes as C
    import paper_2507_17307_amd as P
    shape = W.TINY_S
    w = W.make_weights(shape, seed=9, role=0).to("cuda")
    with pytest.raises(P.RsError):
        P.PagedModel(w, max_ctx=64, n_pages=4, page_size=24)
    m = P.PagedModel(w, max_ctx=64, n_pages=4, page_size=16, max_seqs=2)
    for field, value, word in (("head_dim", 64, "head_dim"), ("n_slots", 1, "slots"), ("max_pages", 3, "max_ctx"), ("n_kv_heads", 4, "n_kv_heads"), ("k", None, "null")):
        kv = P.binding._RsPagedKv.from_buffer_copy(m.cache_struct)
        setattr(kv, field, value)
        assert P.rs_paged_workspace_bytes(m.cfg, kv) == 0 and word in P.rs_last_error()
        with pytest.raises(P.RsError):
            P.rs_create_model_paged(m.cfg, w, kv, m.workspace)
    assert P.rs_paged_workspace_bytes(m.cfg, m.cache_struct) > P.rs_workspace_bytes(m.cfg)
    with pytest.raises(P.RsError, match="smaller"):
        P.rs_create_model_paged(m.cfg, w, m.cache_struct, m.workspace[:-256])
    m.close()
