"""A captured rs_paged_append writes every value that the call itself writes, and no other."""
import pytest
import torch

import paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_replay_writes_the_same_pages(dtype):
    import paper_2507_17307_amd as P
    pg = paged.Pages([5, 1, 70], [14, 40, 100], 2, 64, 16, seed=72).gpu()
    x = torch.randn(pg.rows, 8, 64, generator=pg.gen).to(dtype).cuda()
    f, amp = P.rs_rope_frequencies(64, 1e4)
    r = P.Rope(f.cuda())
    out = torch.empty(pg.rows, 4, 64, dtype=dtype, device="cuda")

    def call():
        P.rs_paged_append(pg.cache, pg.n, pg.rows, pg.dslot, pg.doff, pg.dpos, r, x[:, :4], x[:, 4:6], x[:, 6:], out)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        pg.dpos.sub_(3)
        x.mul_(1.5)
        both = []
        for go in (call, graph.replay):
            for t in (out, pg.dk, pg.dv):
                t.fill_(9.0)
            go()
            torch.cuda.synchronize()
            both.append([t.clone() for t in (out, pg.dk, pg.dv)])
        assert all(torch.equal(a, b) for a, b in zip(*both))
        # (a normal value times 1.5^k that is 9 exactly in every channel of a place there is not)
        held = (both[0][1] != 9.0).any(3).any(1)
        assert int(held.sum()) == pg.rows and int((both[0][2] != 9.0).any(2).any(1).sum()) == pg.rows
