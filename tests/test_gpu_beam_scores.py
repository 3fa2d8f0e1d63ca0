"""Scores of rs_beam_select in double: what a search of many steps needs to tell its beams apart, and logits of any size."""
import math

import pytest
import torch

import beam
import workloads as W
from test_gpu_beam_search import tokens

pytestmark = pytest.mark.gpu

# Of a score after one call: the exponentials' 1.1e-12, up to 2^18 additions of positive numbers (2^18 2^-53 < 3e-11) in ln Z, a few roundings of numbers below 2^20
# (2^-33 each): 1e-9 covers it, and the roundings of the 64-bit loop beside it.
STEP = 1e-9


def run(x, groups, beams, score, n_out, scale=None, last=None, eos=-1, alpha=0.0, length=None):
    """(parent, token, score, length, flags) of the call with double scores, on the CPU."""
    import paper_2507_17307_amd as P
    def dev(t):
        return None if t is None else t.cuda()
    n = groups * n_out
    parent, token, out_len = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
    out, flag = torch.full((n,), 77.0, dtype=torch.float64, device="cuda"), torch.zeros(groups * beams, dtype=torch.int32, device="cuda")
    scratch = torch.full((P.rs_beam_select_scratch_bytes(groups, beams, x.shape[1], n_out),), 255, dtype=torch.uint8, device="cuda")
    P.rs_beam_select(dev(x), groups, beams, dev(scale), dev(score), dev(last), eos, alpha, dev(length), n_out, parent, token, out, out_len if length is not None else None, scratch, flag)
    torch.cuda.synchronize()
    return parent.cpu(), token.cpu(), out.cpu(), out_len.cpu(), flag.cpu()


def compare(x, groups, beams, score, n_out, **more):
    got, want = run(x, groups, beams, score, n_out, **more), beam.select(x, groups, beams, score, n_out, **more)
    assert got[0].tolist() == want[0] and got[1].tolist() == want[1]
    assert torch.equal(got[2] == -math.inf, want[2] == -math.inf)
    fine = want[2] > -math.inf
    assert not bool(fine.any()) or float((got[2] - want[2])[fine].abs().max()) <= STEP
    if more.get("length") is not None:
        assert got[3].tolist() == want[3]
    assert {r for r, f in enumerate(got[4].tolist()) if f} == want[4]
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups, beams, vocab, n_out", [(1, 1, 1, 1), (1, 1, 1, 3), (3, 5, 7, 5), (2, 64, 9, 64), (1, 4, 65, 4), (2, 4, 257, 8), (2, 3, 1025, 12), (1, 4, 50257, 64), (33, 1, 3001, 1)])
def test_sizes(groups, beams, vocab, n_out, dtype):
    g = torch.Generator().manual_seed(groups * 1000 + vocab + n_out)
    x, rows = (torch.randn(groups * beams, vocab, generator=g) * 3).to(dtype), groups * beams
    score, scale = -300 * torch.rand(1, generator=g, dtype=torch.float64) - 4 * torch.rand(rows, generator=g, dtype=torch.float64), torch.rand(rows, generator=g) + 0.5
    compare(x, groups, beams, score, n_out, scale=scale)
    last, length = torch.randint(0, 4, (rows,), generator=g).to(torch.int32), torch.randint(0, 30, (rows,), generator=g).to(torch.int32)
    compare(x, groups, beams, score, n_out, scale=scale, last=last, eos=0, alpha=0.7, length=length)


def test_rows_that_are_bad_or_not_there():
    g = torch.Generator().manual_seed(1)
    x, score = torch.randn(8, 900, generator=g), -torch.rand(8, generator=g, dtype=torch.float64)
    score[1], score[2], score[3], score[4] = math.nan, math.inf, -math.inf, -1e300
    x[5, 3] = math.nan
    got = compare(x, 1, 8, score, 64)
    assert got[4].tolist() == [0, 16, 16, 0, 0, 8, 0, 0]
    compare(x, 8, 1, score, 2)                                                # (-1e300 is no end of the range)


@pytest.mark.parametrize("alpha", [0.0, 0.7, 30.0])
def test_an_ended_beams_score_stays_bit_by_bit(alpha):
    g = torch.Generator().manual_seed(2)
    x, score = torch.randn(64, 300, generator=g), -500 * torch.rand(64, generator=g, dtype=torch.float64) - 1e-3
    score[7], score[8] = -1e-300, -5e-324
    length = torch.randint(0, 2**31 - 2, (64,), generator=g).to(torch.int32)
    got = run(x, 1, 64, score, 64, last=torch.full((64,), 5, dtype=torch.int32), eos=5, alpha=alpha, length=length)
    assert sorted(got[0].tolist()) == list(range(64)) and torch.equal(got[2], score[got[0].long()]) and torch.equal(got[3], length[got[0].long()])
    fp32 = score.float()
    import paper_2507_17307_amd as P
    out, ints = torch.zeros(64, device="cuda"), [torch.zeros(64, dtype=torch.int32, device="cuda") for _ in range(3)]
    scratch = torch.zeros(P.rs_beam_select_scratch_bytes(1, 64, 300, 64), dtype=torch.uint8, device="cuda")
    P.rs_beam_select(x.cuda(), 1, 64, None, fp32.cuda(), torch.full((64,), 5, dtype=torch.int32).cuda(), 5, alpha, length.cuda(), 64, ints[0], ints[1], out, ints[2], scratch)
    assert torch.equal(out.cpu(), fp32[ints[0].cpu().long()])


def log_p(x, scale):
    """ln of the shares of e^(scale x), in 64 bits, with the largest taken out first: right for finite logits of any size."""
    x = x.double() * scale
    x = x - x.max()
    return x - x.exp().sum().log()


@pytest.mark.parametrize("dtype, low", [(torch.float32, torch.finfo(torch.float32).min), (torch.bfloat16, torch.finfo(torch.bfloat16).min), (torch.float32, -1e30), (torch.float32, 3e38), (torch.float32, -65504.0)])
@pytest.mark.parametrize("scale", [1.0, 0.37])
def test_masks_of_the_lowest_value(dtype, low, scale):
    """A row whose mask leaves nothing has tokens of log probability -ln vocab each, not 0, so that it does not win; one of two values has the larger ones' share."""
    vocab = 3001
    x = torch.full((4, vocab), low).to(dtype)
    x[0, 17], x[0, 40] = max(1.0, low * 0.5), 0.5
    x[2, 1000:] = float(x[2, 0]) / 2
    x[3] = torch.randn(vocab, generator=torch.Generator().manual_seed(3)).to(dtype)
    score = torch.tensor([-20.0, -1.0, -3.0, -1.5], dtype=torch.float64)
    got = run(x, 1, 4, score, 12, scale=torch.full((4,), scale))
    found = sorted((-float(s + p), b, at, t) for b, s in enumerate(score) for row in [log_p(x[b], float(torch.tensor(scale)))]
                   for at, t in enumerate(torch.sort(x[b].float(), descending=True, stable=True).indices[:12].tolist()) for p in [row[t]])[:12]
    assert got[0].tolist() == [f[1] for f in found] and got[1].tolist() == [f[3] for f in found]
    assert max(abs(float(a) + f[0]) for a, f in zip(got[2], found)) <= STEP
    assert not bool(got[4].any())


def near(groups, vocab, steps):
    """Logits of every step: a token of 40 percent and 3000 others; where a coin falls so, the second beam's is likelier by 2^-19, or one step of it."""
    g = torch.Generator().manual_seed(groups + vocab + steps)
    x = torch.randn(steps, groups, 1, vocab, generator=g) * 0.1
    best = torch.randint(0, vocab, (steps, groups, 1, 1), generator=g)
    x.scatter_(3, best, 7.0 + torch.rand(steps, groups, 1, 1, generator=g))
    x = x.repeat(1, 1, 2, 1)
    up = (torch.rand(steps, groups, 1, 1, generator=g) < 0.3).float() * 2.0 ** -19
    second = x[:, :, 1:]
    second.scatter_(3, best, second.gather(3, best) + up)
    return x.view(steps, groups * 2, vocab)


def follow(x, groups, score, rounded):
    """Parents and tokens of every step and the scores behind the last one, by the 64-bit loop; rounded: to fp32 between the steps."""
    lines = []
    for rows in x:
        parent, token, score, _, _ = beam.select(rows, groups, 2, score, 2)
        if rounded:
            score = score.float().double()
        lines.append((parent, token))
    return lines, score


def test_beams_nearer_than_fp32_over_many_steps():
    """Scores fall to some -400, where a step of fp32 is 3e-5; the beams of a group are some 1e-6 apart and pass each other now and then."""
    import paper_2507_17307_amd as P
    groups, vocab, steps = 3, 3000, 400
    x = near(groups, vocab, steps)
    begin = torch.tensor([0.0, -3e-7, -10.0, -10.0 - 1e-6, -3.0, -3.0 - 4e-7], dtype=torch.float64)
    want, end = follow(x, groups, begin, False)
    assert sum(p[:2] == [1, 0] for p, _ in want) > 20 and float(end.max()) < -300 and float((end[::2] - end[1::2]).max()) < 2.0 ** -16
    assert follow(x, groups, begin, True)[0] != want
    rows, xs = groups * 2, x.cuda()
    score, parent, token = begin.cuda(), torch.zeros(steps, rows, dtype=torch.int32, device="cuda"), torch.zeros(steps, rows, dtype=torch.int32, device="cuda")
    scratch = torch.zeros(P.rs_beam_select_scratch_bytes(groups, 2, vocab, 2), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        P.rs_beam_select(xs[step], groups, 2, None, score, None, -1, 0.0, None, 2, parent[step], token[step], score, None, scratch)
    torch.cuda.synchronize()
    assert list(zip(parent.tolist(), token.tolist())) == want
    assert float((score.cpu() - end).abs().max()) <= STEP * steps


def test_a_search_adds_its_scores_up_in_double(monkeypatch):
    """Each reply's score is the sum of its tokens' log probabilities under the logits that the search saw."""
    import paper_2507_17307_amd as P
    w = W.make_weights(W.TINY_L, seed=9, role=0).to("cuda")
    model, seen = P.PagedModel(w, max_ctx=160, n_pages=200, page_size=16, max_seqs=12, max_rows=12), []
    select = P.binding.rs_beam_select

    def watched(logits, *args):
        seen.append(logits.double().clone())
        select(logits, *args)
    monkeypatch.setattr(P.binding, "rs_beam_select", watched)

    class Traced(P.BeamSearch):
        def _read(self, parents, tokens, scores):
            self.trace = parents, tokens
            return super()._read(parents, tokens, scores)
    search = Traced(model, 2, 6, logit_scale=0.5)
    got = search.generate([tokens(W.TINY_L, n, 60 + n) for n in (7, 20)], 120)
    torch.cuda.synchronize()
    for g in range(2):
        for b in range(6):
            at, total = b, 0.0
            for step in range(119, -1, -1):
                r = 6 * g + at
                at = search.trace[0][step][r]
                total += float(torch.log_softmax(seen[step][6 * g + at] * 0.5, 0)[search.trace[1][step][r]])
            assert total < -100 and abs(got[g][b].score - total) <= 120 * STEP
    model.close()


def test_calls_of_both_score_types_replayed_side_by_side():
    """Two captured calls, one with double and one with fp32 scores, in place, replayed on two streams at once; every replay against the 64-bit loop of what it started from."""
    import paper_2507_17307_amd as P
    g = torch.Generator().manual_seed(21)
    x = [torch.randn(12, 30011, generator=g).cuda() * 3 for _ in range(2)]
    scores = [(-400 * torch.rand(12, generator=g, dtype=torch.float64)).to(t).cuda() for t in (torch.float64, torch.float32)]
    states = [(torch.ones(12, dtype=torch.int32).cuda(), torch.full((12,), 9, dtype=torch.int32).cuda(), torch.zeros(12, dtype=torch.int32).cuda(),
               torch.full((P.rs_beam_select_scratch_bytes(3, 4, 30011, 4),), 255, dtype=torch.uint8).cuda()) for _ in range(2)]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for logits, score, (last, length, parent, scratch), stream in zip(x, scores, states, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            P.rs_beam_select(logits, 3, 4, None, score, last, 5, 0.5, length, 4, parent, last, score, length, scratch)
        graphs.append(graph)
    for step in range(4):
        for logits in x:
            logits.mul_(0.9).add_(torch.randn(12, 1, generator=g).cuda())
        wants = [beam.select(logits.cpu(), 3, 4, score.cpu(), 4, last=s[0].cpu(), eos=5, alpha=0.5, length=s[1].cpu()) for logits, score, s in zip(x, scores, states)]
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for k, (want, score, s) in enumerate(zip(wants, scores, states)):
            assert s[2].tolist() == want[0] and s[0].tolist() == want[1] and s[1].tolist() == want[3], (step, k)
            if k == 0:
                assert float((score.cpu() - want[2]).abs().max()) <= STEP
            else:
                beam.check_scores(score, want[2])
