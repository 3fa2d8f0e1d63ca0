"""rs_beam_select against plain loops in 64 bits: types, sizes, strides, masks, ends, lengths, ties, refusals of rows."""
import math

import pytest
import torch

import beam

pytestmark = pytest.mark.gpu


def run(logits, n_groups, n_beams, score, n_out, scale=None, last=None, eos=-1, alpha=0.0, length=None, flags=True):
    """(parent, token, score, length, flags) of the call, on the CPU."""
    import paper_2507_17307_amd as P
    def dev(t):
        return None if t is None else t.cuda()
    n = n_groups * n_out
    parent, token, out_len = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
    out = torch.full((n,), 77.0, device="cuda")
    flag = torch.zeros(n_groups * n_beams, dtype=torch.int32, device="cuda") if flags else None
    scratch = torch.full((P.rs_beam_select_scratch_bytes(n_groups, n_beams, logits.shape[1], n_out),), 255, dtype=torch.uint8, device="cuda")
    P.rs_beam_select(logits if logits.is_cuda else logits.cuda(), n_groups, n_beams, dev(scale), dev(score), dev(last), eos, alpha, dev(length), n_out, parent, token, out,
                     out_len if length is not None else None, scratch, flag)
    torch.cuda.synchronize()
    return parent.cpu(), token.cpu(), out.cpu(), out_len.cpu(), None if flag is None else flag.cpu()


def compare(logits, n_groups, n_beams, score, n_out, what="", **more):
    got = run(logits, n_groups, n_beams, score, n_out, **more)
    want = beam.select(logits.cpu(), n_groups, n_beams, score, n_out, **more)
    assert got[0].tolist() == want[0] and got[1].tolist() == want[1], what
    beam.check_scores(got[2], want[2], what)
    if more.get("length") is not None:
        assert got[3].tolist() == want[3], what
    assert {r for r, f in enumerate(got[4].tolist()) if f} == want[4], what
    return got


def normal(seed, rows, vocab, dtype=torch.float32, std=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g) * std).to(dtype), -torch.rand(rows, generator=g) * 5 - 1, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups, beams, vocab, n_out", [
    (1, 1, 1, 1), (1, 1, 1, 3), (1, 2, 2, 4), (3, 5, 7, 5), (2, 64, 9, 64), (1, 1, 63, 64), (2, 3, 64, 64), (1, 4, 65, 4), (4, 2, 255, 2), (2, 4, 257, 8), (1, 3, 1023, 3),
    (5, 4, 1024, 4), (2, 6, 1025, 12), (1, 4, 4095, 5), (3, 2, 4100, 33), (2, 4, 16387, 4), (1, 7, 50257, 7), (1, 4, 152064, 64), (33, 1, 3001, 1), (1, 64, 2049, 64)])
def test_sizes(groups, beams, vocab, n_out, dtype):
    x, score, g = normal(groups * 1000 + vocab + n_out, groups * beams, vocab, dtype)
    scale = torch.rand(groups * beams, generator=g) + 0.5
    compare(x, groups, beams, score, n_out, scale=scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab, spare, first", [(1000, 1, 0), (1000, 8, 3), (1001, 7, 1), (2047, 5, 2), (6000, 13, 5), (40001, 3, 7)])
def test_strides_and_addresses(vocab, spare, first, dtype):
    x, score, g = normal(vocab + first, 6, vocab + spare + first, dtype)
    # (what lies around a row would win if it were looked at)
    wide = torch.full((6, first + vocab + spare), 1e4, dtype=dtype)
    wide[:, first:first + vocab] = x[:, :vocab]
    view = wide.cuda()[:, first:first + vocab]
    compare(view, 2, 3, score, 6)


@pytest.mark.parametrize("vocab", [130, 5000, 70001])
def test_masks_leave_few_or_no_tokens(vocab):
    x, score, g = normal(vocab, 12, vocab)
    x.masked_fill_(torch.rand(12, vocab, generator=g) < 0.99, -math.inf)
    x[3] = -math.inf
    x[6:9] = -math.inf                                                    # a whole group
    x[9:12] = -math.inf
    x[10, vocab - 1] = 0.25                                               # a group with one candidate
    got = compare(x, 4, 3, score, 8)
    assert got[0][16:24].tolist() == [-1] * 8 and got[0][24:32].tolist() == [1] + [-1] * 7 and got[1][24] == vocab - 1


def test_masks_of_the_lowest_value_are_candidates():
    low = torch.finfo(torch.float32).min
    x = torch.full((4, 3001), low)
    x[0, 17], x[1, 3000], x[2, 0], x[2, 1] = 1.0, 2.0, low / 2, -1e30
    compare(x, 2, 2, torch.tensor([-1.0, -2.0, -3.0, -4.0]), 4)


def test_equal_logits_go_to_the_lowest_token_and_beam():
    x = torch.zeros(4, 20000)
    got = compare(x, 1, 4, torch.tensor([-2.0, -1.0, -1.0, -3.0]), 10)
    assert got[0].tolist() == [1] * 10 and got[1].tolist() == list(range(10))
    x[:, 12345] = 3.0
    x[:, 19999] = 3.0
    got = compare(x, 1, 4, torch.tensor([-2.0, -1.0, -1.0, -3.0]), 7)
    assert got[0].tolist() == [1, 1, 2, 2, 0, 0, 3] and got[1].tolist() == [12345, 19999] * 3 + [12345]


def test_zero_and_minus_zero_are_equal():
    x = torch.full((1, 300), -5.0)
    x[0, 100], x[0, 50], x[0, 200] = 0.0, -0.0, 0.0
    assert run(x, 1, 1, torch.zeros(1), 3)[1].tolist() == [50, 100, 200]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_in_order_and_against_it(dtype):
    x = torch.linspace(-20, 20, 30011).to(dtype)
    x = torch.stack([x, x.flip(0), x, x.flip(0)])
    compare(x, 2, 2, torch.tensor([-1.0, -1.5, -7.0, -6.5]), 24)


@pytest.mark.parametrize("n_out", [1, 16, 64])
def test_all_large_values_in_one_stretch(n_out):
    x, score, g = normal(5, 2, 33000)
    x[0, 5000:5400] += 40.0                                               # more of them than any list of candidates holds
    x[1, 31900:33000] = 50.0
    compare(x, 1, 2, score, n_out)
    compare(x, 2, 1, score, n_out)


def test_ends_lengths_and_penalties():
    x, score, g = normal(8, 24, 1500)
    last = torch.randint(0, 4, (24,), generator=g).to(torch.int32)
    length = torch.randint(0, 30, (24,), generator=g).to(torch.int32)
    for alpha in (0.0, 0.6, 1.0, 2.5):
        compare(x, 4, 6, score, 6, last=last, eos=2, alpha=alpha, length=length, what=str(alpha))
        compare(x, 6, 4, score, 9, last=last, eos=2, alpha=alpha, length=length, what=str(alpha))
    compare(x, 4, 6, score, 6, last=last, eos=-1, length=length)
    everything_ended = torch.full((24,), 2, dtype=torch.int32)
    got = compare(x, 4, 6, score, 8, last=everything_ended, eos=2, alpha=1.0, length=length)
    assert got[0][6:8].tolist() == [-1, -1] and set(got[1][:6].tolist()) == {2}


def test_rows_that_are_not_read_may_hold_anything():
    x, score, g = normal(9, 6, 5000)
    score[1], x[1] = -math.inf, math.nan
    last = torch.tensor([0, 0, 0, 0, 5, 0], dtype=torch.int32)
    x[4] = math.nan
    got = compare(x, 2, 3, score, 4, last=last, eos=5)
    assert not got[4].any()
    compare(x, 2, 3, torch.full((6,), -math.inf), 4)


def test_bad_rows_are_flagged_and_have_no_candidates():
    x, score, g = normal(10, 8, 9001)
    x[0, 9000], x[1, 0], x[2, 4444] = math.nan, math.inf, -math.inf
    score[3], score[4] = math.nan, math.inf
    scale = torch.ones(8)
    scale[5], scale[6], scale[7] = 0.0, -1.0, math.inf
    got = compare(x, 1, 8, score, 5, scale=scale)
    assert got[4].tolist() == [8, 8, 0, 16, 16, 16, 16, 16] and set(got[0].tolist()) == {2}
    length = torch.tensor([1, 1, 1, 1, 1, 1, 1, -1], dtype=torch.int32)
    compare(x, 2, 4, score, 5, length=length, alpha=1.0)
    length[2] = 2**31 - 1
    compare(x, 2, 4, score, 5, length=length, alpha=1.0)
    assert run(x, 1, 8, score, 5, scale=scale, flags=False)[0].tolist() == got[0].tolist()


@pytest.mark.parametrize("big", [88.0, 1e4, 3e38])
def test_large_logits(big):
    x, score, g = normal(11, 4, 2500)
    x[0, 7], x[0, 8], x[1, 100], x[2] = big, big * 0.999, -big, -big
    compare(x, 2, 2, score, 6)


def test_neighbours_that_32_bits_do_not_tell_apart():
    """Two beams whose best continuations are 2^-30 apart, in either order, below scores whose steps are 2^-17."""
    x = torch.full((2, 4000), -30.0)
    x[:, 11] = 0.0
    score = torch.tensor([-100.0, -100.0])
    for up in (0, 1):
        y = x.clone()
        y[up, 12] = math.log(2.0 ** -30)                                  # the beam's ln Z grows by 2^-30
        got = run(y, 1, 2, score, 2)
        assert got[0].tolist() == [1 - up, up] and got[1].tolist() == [11, 11]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_batches_a_wave(dtype):
    """64 x 64 candidates leave a row one workgroup: 13 batches a wave, whose logits rise past what one exponent serves (2^500 above the first), and past
    the size up to which they are added up in that way at all."""
    x, score, g = normal(13, 64, 50257, dtype)
    x[1, 30000:] += 1000.0
    x[2, 9000:40000] += 2000.0
    x[3, 20000] = 3500.0
    x[4, 13000:] -= 2500.0
    x[5] *= 500.0
    x[6, 100:50000] = -math.inf
    x[7, 5000:] = -math.inf
    x[8] -= 1000.0
    x[9, 50256] = 90.0
    compare(x, 1, 64, score, 64)
    compare(x, 1, 64, score * 0, 64, scale=torch.rand(64, generator=g) * 2 + 0.1)


def test_thousands_of_equal_candidates():
    x = torch.zeros(128, 300)
    got = compare(x, 2, 64, torch.full((128,), -1.0), 64)
    assert got[0].tolist() == [0] * 128 and got[1].tolist() == list(range(64)) * 2
    score = torch.full((128,), -1.0)
    score[:40] = -3.0                                                         # (3000 equals from beam 40 on, others below them)
    x[70, 5] = 1.0
    compare(x, 2, 64, score, 64)


def test_scores_far_apart_and_beams_that_are_not_there():
    x, score, g = normal(14, 64, 4000)
    score[:] = -torch.arange(64) * 40.0
    score[::4] = -math.inf
    compare(x, 1, 64, score, 64)
    compare(x, 2, 32, score.flip(0), 32)
    score[:] = -math.inf
    score[0], score[32] = 0.0, 0.0                                            # a search's first step
    compare(x, 2, 32, score, 64)


def test_two_calls_at_once():
    import paper_2507_17307_amd as P
    calls = []
    for k in range(2):
        x, score, g = normal(20 + k, 24, 100003)
        out = [torch.zeros(48, dtype=torch.int32, device="cuda") for _ in range(2)] + [torch.zeros(48, device="cuda")]
        calls.append((x.cuda(), score.cuda(), out, torch.empty(P.rs_beam_select_scratch_bytes(6, 4, 100003, 8), dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), x, score))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, score, out, scratch, stream, _, _ in calls:
            P.rs_beam_select(x, 6, 4, None, score, None, -1, 0.0, None, 8, out[0], out[1], out[2], None, scratch, stream=stream)
    torch.cuda.synchronize()
    for _, _, out, _, _, x, score in calls:
        want = beam.select(x, 6, 4, score, 8)
        assert out[0].tolist() == want[0] and out[1].tolist() == want[1]
        beam.check_scores(out[2], want[2])


@pytest.mark.parametrize("scale", [1e-30, 1e-34, 1e-36, 1e-40, 1e-45])
def test_scales_next_to_nothing(scale):
    """All tokens but the masked ones are equally likely."""
    x, score, g = normal(15, 4, 5003)
    x[0, ::2] = -math.inf
    x[1, 1:] = -math.inf
    x[2, :5000] = -math.inf
    compare(x, 2, 2, score, 6, scale=torch.full((4,), scale))


def test_in_place_and_replayed():
    import paper_2507_17307_amd as P
    x, score, g = normal(12, 12, 60000)
    x = x.cuda()
    state = [score.cuda(), torch.ones(12, dtype=torch.int32).cuda(), torch.full((12,), 9, dtype=torch.int32).cuda()]
    parent = torch.zeros(12, dtype=torch.int32, device="cuda")
    scratch = torch.zeros(P.rs_beam_select_scratch_bytes(3, 4, 60000, 4), dtype=torch.uint8, device="cuda")

    def call():
        P.rs_beam_select(x, 3, 4, None, state[0], state[1], 5, 0.5, state[2], 4, parent, state[1], state[0], state[2], scratch)
    begin = [t.clone() for t in state]
    call()
    torch.cuda.synchronize()
    for t, b in zip(state, begin):
        t.copy_(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        x.mul_(0.9).add_(torch.randn(12, 1, generator=g).cuda())
        before = [t.cpu() for t in state]
        want = beam.select(x.cpu(), 3, 4, before[0], 4, last=before[1], eos=5, alpha=0.5, length=before[2])
        graph.replay()
        torch.cuda.synchronize()
        assert parent.tolist() == want[0] and state[1].tolist() == want[1] and state[2].tolist() == want[3]
        beam.check_scores(state[0], want[2])
        after = [t.clone() for t in state]
        for t, b in zip(state, before):
            t.copy_(b.cuda())
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(after, state))
