"""rs_rope_rows against 64 bits: both pairings, part of the head, far positions, scaled frequencies, strides, in place, the inverse, gradients."""
import pytest
import torch

import paged

pytestmark = pytest.mark.gpu


def make(rows, heads, hd, dtype, seed, top=200000):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, top, (rows,), generator=g).to(torch.int32)
    pos[0] = 0
    pos[-1] = 2 ** 31 - 1 if rows > 1 else 4570                    # as far as a position goes
    return torch.randn(rows, heads, hd, generator=g).to(dtype), pos


def rope(rot, interleaved=False, kind=0, factor=1.0):
    import paper_2507_17307_amd as P
    f, amp = P.rs_rope_frequencies(rot, 1e6, kind, factor)
    return f, amp, P.Rope(f.cuda(), interleaved, amp)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,hd,rot", [(1, 1, 8, 8), (1, 12, 128, 128), (3, 28, 128, 64), (65, 5, 64, 48), (130, 8, 32, 24), (2049, 3, 128, 128), (5, 2, 1024, 1000), (4099, 1, 256, 8)])
def test_rows_are_rotated(rows, heads, hd, rot, interleaved, dtype):
    import paper_2507_17307_amd as P
    x, pos = make(rows, heads, hd, dtype, rows * 7 + rot)
    f, amp, r = rope(rot, interleaved, 2, 4.0)
    for inverse in (False, True):
        out = torch.full_like(x, 7.0, device="cuda")
        P.rs_rope_rows(r, pos.cuda(), x.cuda(), out, inverse=inverse)
        paged.close(out.cpu(), *paged.turned(x, pos, f, amp, interleaved, inverse), f"inverse {inverse}")


def test_negative_positions_and_special_values():
    import paper_2507_17307_amd as P
    x, pos = make(6, 2, 64, torch.float32, 3)
    pos = -pos.clamp(max=100000)
    x[2, 1, 5], x[3, 0, 60] = float("nan"), float("inf")
    f, amp, r = rope(64, False)
    out = torch.empty_like(x, device="cuda")
    P.rs_rope_rows(r, pos.cuda(), x.cuda(), out)
    want, err = paged.turned(x, pos, f, amp)
    keep = torch.isfinite(want)
    assert (~keep).sum() == 4 and torch.equal(torch.isfinite(out.cpu()), keep)
    paged.close(out.cpu()[keep], want[keep], err[keep])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_rows_in_place_leave_the_rest_alone(dtype):
    import paper_2507_17307_amd as P
    x, pos = make(37, 10, 64, dtype, 5)
    f, amp, r = rope(64, True)
    buf = x.cuda()
    view = buf[:, 2:7]                                            # heads of a fused projection's rows
    P.rs_rope_rows(r, pos.cuda(), view, view)
    got = buf.cpu()
    paged.close(got[:, 2:7], *paged.turned(x[:, 2:7], pos, f, amp, True))
    assert torch.equal(got[:, :2], x[:, :2]) and torch.equal(got[:, 7:], x[:, 7:])


def test_the_inverse_is_the_gradient():
    """The rotation is linear in x: the gradient of sum(g * out) is the inverse applied to g, and differences of the forward pass show the same."""
    import paper_2507_17307_amd as P
    x, pos = make(9, 3, 128, torch.float32, 8, top=3000)
    pos[-1] = 2999
    g = torch.randn(x.shape, generator=torch.Generator().manual_seed(9))
    f, amp, r = rope(96, False, 2, 2.0)
    grad = torch.empty_like(x, device="cuda")
    P.rs_rope_rows(r, pos.cuda(), g.cuda(), grad, inverse=True)
    paged.close(grad.cpu(), *paged.turned(g, pos, f, amp, False, True), "formula")
    d = torch.randn(x.shape, generator=torch.Generator().manual_seed(10))
    up, down = torch.empty_like(grad), torch.empty_like(grad)
    P.rs_rope_rows(r, pos.cuda(), (x + d).cuda(), up)
    P.rs_rope_rows(r, pos.cuda(), (x - d).cuda(), down)
    have = float((g.double() * (up.cpu().double() - down.cpu().double())).sum() / 2)
    want = float((grad.cpu().double() * d.double()).sum())
    # 3456 products, each with the errors of `turned` on magnitudes of about 2 x 2: 2^-20 apiece
    assert abs(have - want) <= x.numel() * 4 * 2.0 ** -20


def test_a_captured_rotation_follows_its_inputs_and_another_stream_gives_the_same():
    import paper_2507_17307_amd as P
    x, pos = make(33, 4, 128, torch.bfloat16, 11)
    f, amp, r = rope(128)
    dx, dpos, out = x.cuda(), pos.cuda(), torch.empty_like(x, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.rs_rope_rows(r, dpos, dx, out)
    s.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.rs_rope_rows(r, dpos, dx, out)
    for k in range(3):
        if k:
            dpos.add_(17)
        want = torch.empty_like(out)
        P.rs_rope_rows(r, dpos, dx, want)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and (k or torch.equal(out, first))
