"""rs_paged_attention against 64 bits: decode, chunks and mixtures, head layouts, windows, pages that end inside a tile, values that no row sees."""
import math

import pytest
import torch

import paged

pytestmark = pytest.mark.gpu


def call(pg, q, scale, window=0, pad=0, off=True, flags=None, out=None, lse=None):
    import paper_2507_17307_amd as P
    rows, nq = q.shape[0], q.shape[1]
    dq = q.cuda()
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full((rows, nq), 9.0, device="cuda") if lse is None else lse
    size = P.rs_paged_attention_scratch_bytes(pg.cache, pg.n, rows, nq)
    scratch = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    P.rs_paged_attention(pg.cache, pg.n, rows, pg.dslot, pg.doff if off else None, pg.dpos, dq, scale, window, out, lse, scratch, flags)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


def check(pg, q, scale, window, out, lse):
    want, z, eo, ez = paged.attention(pg, q[:pg.rows], scale, window)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(out[:pg.rows]), torch.isnan(want)) and torch.equal(torch.isinf(out[:pg.rows]), torch.isinf(want))
    paged.close(out[:pg.rows][fine], want[fine], eo[fine], "out")
    fine = torch.isfinite(z)
    paged.close(lse[:pg.rows][fine], z[fine], ez[fine], "lse")
    assert bool((out[pg.rows:] == 9.0).all()) and bool((lse[pg.rows:] == 9.0).all())


CASES = [  # spans, positions held before, query heads, KV heads, channels, page, window
    ([1], [0], 1, 1, 32, 16, 0),
    ([1], [200], 12, 2, 128, 64, 0),
    ([1], [4561], 28, 4, 128, 64, 0),
    ([1, 1, 1, 1, 1, 1, 1], [0, 1, 15, 16, 31, 700, 2050], 28, 4, 128, 16, 0),
    ([1] * 40, [i * 53 for i in range(40)], 16, 1, 64, 32, 0),
    ([1] * 9, [i * 300 for i in range(9)], 8, 8, 32, 1024, 100),
    ([2, 5, 1, 3], [1000, 17, 130, 0], 12, 2, 128, 64, 0),
    ([7, 0, 30, 1, 64], [0, 9, 50, 640, 127], 6, 2, 64, 16, 33),
    ([61], [900], 40, 8, 128, 128, 0),
    ([130, 1, 257], [0, 2000, 300], 14, 2, 128, 64, 0),
    ([300], [0], 16, 4, 64, 16, 1),
    ([200, 90], [511, 64], 5, 5, 128, 32, 190),
    ([700], [33], 3, 1, 32, 256, 0),
    ([96, 1, 1, 1], [64, 63, 64, 65], 30, 2, 64, 64, 64),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_matches_64_bits(case, dtype):
    spans, pos0, nq, nkv, hd, page, window = CASES[case]
    pg = paged.Pages(spans, pos0, nkv, hd, page, seed=case, fill=float("nan")).gpu()
    pad = 3 if sum(spans) > len(spans) else 0
    q = torch.randn(pg.rows + pad, nq, hd, generator=pg.gen).to(dtype)
    out, lse = call(pg, q, hd ** -0.5, window)
    check(pg, q, hd ** -0.5, window, out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("spans,pos0", [([1, 1], [300, 64]), ([40, 3], [70, 5])])
def test_sharp_and_shifted_scores(spans, pos0, dtype):
    """Scores of hundreds, of both signs: the running maximum carries the sums, nothing overflows."""
    pg = paged.Pages(spans, pos0, 2, 64, 16, seed=30).gpu()
    q = (torch.randn(pg.rows, 6, 64, generator=pg.gen) * 12).to(dtype)
    out, lse = call(pg, q, 0.7)
    check(pg, q, 0.7, 0, out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("spans,pos0", [([1], [90]), ([50], [90]), ([200], [0])])
def test_what_a_row_does_not_see_does_not_reach_it(spans, pos0, window, dtype):
    """NaN and infinities in K and V of one position: the rows that see it have them, the others, of the same tile too, do not."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        pg = paged.Pages(spans, pos0, 1, 128, 16, seed=31)
        p = pos0[0] + spans[0] // 2
        for at, chan in ((p, 7), (p - 30, 100)):
            pg.v[pg.table[pg.slot[0], at // 16], 0, chan, at % 16] = bad
        if math.isnan(bad):
            pg.k[pg.table[pg.slot[0], (p + 1) // 16] if p + 1 < pos0[0] + spans[0] else 0, 0, (p + 1) % 16, 3] = bad
        pg.gpu()
        q = torch.randn(pg.rows, 4, 128, generator=pg.gen).to(dtype)
        out, lse = call(pg, q, 0.1, window)
        check(pg, q, 0.1, window, out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strided_rows_and_no_offsets(dtype):
    pg = paged.Pages([1] * 5, [10, 200, 64, 63, 0], 2, 64, 16, seed=32).gpu()
    wide = torch.randn(7, 14, 64, generator=pg.gen).to(dtype)
    q = wide[:, 2:10]
    out = torch.full((7, 20, 64), 9.0, dtype=dtype, device="cuda")
    got, lse = call(pg, q, 0.125, off=False, out=out[:, 8:16])
    check(pg, q, 0.125, 0, got, lse)
    assert bool((out[:, :8] == 9.0).all()) and bool((out[:, 16:] == 9.0).all())


def test_rows_out_of_range_are_skipped_and_flagged():
    pg = paged.Pages([4, 4, 4, 3, 4], [10, 20, 30, 50, 5], 2, 64, 16, seed=33).gpu()
    q = torch.randn(pg.rows, 6, 64, generator=pg.gen)
    pg.dslot[0] = -5
    pg.dpos[1] = 10 ** 6
    pg.dtable[pg.slot[2].item(), 1] = -7                                      # positions 16 .. 31 of the third sequence
    flags = torch.zeros(5, dtype=torch.int32, device="cuda")
    out, lse = call(pg, q, 0.1, flags=flags)
    assert flags.tolist() == [16, 16, 16, 0, 0]
    assert bool((out[:8] == 9.0).all()) and bool((lse[:8] == 9.0).all())
    want, z, eo, ez = paged.attention(pg, q, 0.1)
    paged.close(out[12:], want[12:], eo[12:])
    paged.close(lse[12:], z[12:], ez[12:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("odd", [False, True])
def test_offsets_that_step_back_are_flagged_and_do_not_disturb_the_others(odd, dtype):
    """Sequences 0, 2 and 4 are the same rows, which brings more blocks than n_rows rows have; sequence 5 is alone in its rows."""
    pg = paged.Pages([400, 3], [100, 30], 2, 64, 16, seed=44)
    if odd:
        pg.v[pg.table[pg.slot[0], 3], 1, 5, 7] = math.nan
    pg.gpu()
    q = torch.randn(pg.rows, 10, 64, generator=pg.gen).to(dtype)
    pg.n = 6
    pg.doff = torch.tensor([0, 400, 0, 400, 0, 400, 403], dtype=torch.int32, device="cuda")
    pg.dslot = pg.dslot[[0, 0, 0, 0, 0, 1]].contiguous()
    pg.dpos = pg.dpos[[0, 0, 0, 0, 0, 1]].contiguous()
    flags = torch.zeros(6, dtype=torch.int32, device="cuda")
    out, lse = call(pg, q, 0.1, flags=flags)
    assert flags.tolist() == [0, 16, 0, 16, 0, 0]
    check(pg, q, 0.1, 0, out, lse)


def test_a_page_that_the_window_has_left_behind_may_be_gone():
    pg = paged.Pages([3, 1], [100, 200], 2, 64, 16, seed=34).gpu()
    q = torch.randn(pg.rows, 6, 64, generator=pg.gen)
    pg.dtable[pg.slot[0].item(), :5] = -1                                     # positions 0 .. 79; the first row sees 81 .. 100
    pg.dtable[pg.slot[1].item(), :11] = 10 ** 6                               # 0 .. 175; 181 .. 200
    flags = torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse = call(pg, q, 0.1, window=20, flags=flags)
    assert flags.tolist() == [0, 0]
    check(pg, q, 0.1, 20, out, lse)


def test_a_cache_of_more_than_4_gib_and_slots_that_repeat():
    """Pages whose elements lie beyond 32 bits; two spans read the same slot."""
    import paper_2507_17307_amd as P
    n_pages, nkv, page, hd = 5000, 4, 1024, 128                               # 5.2 GB a tensor
    k = torch.zeros(n_pages, nkv, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(n_pages, nkv, hd, page, dtype=torch.bfloat16, device="cuda")
    pg = paged.Pages([2, 1], [1500, 2040], nkv, hd, page, seed=35, spare_pages=0).gpu()
    far = [4999, 4100, 4321, 4998][:pg.k.shape[0]]
    k[far], v[far] = pg.dk, pg.dv
    table = torch.tensor([far[i] if i >= 0 else -1 for i in pg.table.flatten().tolist()], dtype=torch.int32, device="cuda").view(pg.table.shape)
    q = torch.randn(pg.rows, 8, hd, generator=pg.gen)
    near, lse = call(pg, q, 0.09)
    check(pg, q, 0.09, 0, near, lse)
    pg.cache = P.PagedCache(k, v, table)
    out, lse2 = call(pg, q, 0.09)
    assert torch.equal(out, near) and torch.equal(lse, lse2)
    pg.dslot[0] = pg.dslot[1]
    out, _ = call(pg, q, 0.09)
    assert torch.equal(out[2], near[2]) and not torch.equal(out[:2], near[:2])


def test_a_captured_call_follows_its_inputs_and_another_stream_gives_the_same():
    import paper_2507_17307_amd as P
    pg = paged.Pages([1] * 6, [300, 64, 63, 0, 1000, 17], 2, 64, 16, seed=36).gpu()
    dq = torch.randn(pg.rows, 6, 64, generator=pg.gen).cuda()
    out, lse = torch.empty_like(dq), torch.empty(pg.rows, 6, device="cuda")
    scratch = torch.empty(P.rs_paged_attention_scratch_bytes(pg.cache, pg.n, pg.rows, 6), dtype=torch.uint8, device="cuda")

    def go(o, z):
        P.rs_paged_attention(pg.cache, pg.n, pg.rows, pg.dslot, None, pg.dpos, dq, 0.1, 0, o, z, scratch)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        go(out, lse)
    s.synchronize()
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(out, lse)
    for i in range(3):
        if i:
            pg.dpos[4] -= 333
            dq.mul_(0.9)
        want, z = torch.empty_like(out), torch.empty_like(lse)
        go(want, z)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, z) and (i or torch.equal(out, first))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_run_of_chunks_and_single_tokens(dtype):
    """The operators together: a prompt in chunks, then tokens one by one, two sequences beside each other in one cache; every call's output is that
    of attention over all rows so far, rotated in 64 bits."""
    import paper_2507_17307_amd as P
    nq, nkv, hd, page, total = 8, 2, 64, 16, [75, 118]
    pg = paged.Pages(total, [0, 0], nkv, hd, page, seed=37).gpu()
    x = [torch.randn(t, nq + 2 * nkv, hd, generator=pg.gen).to(dtype) for t in total]
    f, amp = P.rs_rope_frequencies(hd, 1e4)
    r = P.Rope(f.cuda(), amplitude=amp)
    got = [[], []]
    steps = [(40, 70), (30, 0), (0, 43), (1, 1), (1, 1), (2, 1), (1, 2)]
    at = [0, 0]
    for ms in steps:
        rows = torch.cat([x[b][at[b]:at[b] + ms[b]] for b in (0, 1)]).cuda()
        q, k, v = rows.split([nq, nkv, nkv], 1)
        off = torch.tensor([0, ms[0], sum(ms)], dtype=torch.int32, device="cuda")
        pos = torch.tensor(at, dtype=torch.int32, device="cuda")
        qr, out = torch.empty(sum(ms), nq, hd, dtype=dtype, device="cuda"), torch.empty(sum(ms), nq, hd, dtype=dtype, device="cuda")
        flags = torch.zeros(2, dtype=torch.int32, device="cuda")
        scratch = torch.empty(P.rs_paged_attention_scratch_bytes(pg.cache, 2, sum(ms), nq), dtype=torch.uint8, device="cuda")
        P.rs_paged_append(pg.cache, 2, sum(ms), pg.dslot, off, pos, r, q, k, v, qr, flags)
        P.rs_paged_attention(pg.cache, 2, sum(ms), pg.dslot, off, pos, qr, hd ** -0.5, 0, out, None, scratch, flags)
        assert flags.tolist() == [0, 0]
        got[0].append(out[:ms[0]].cpu())
        got[1].append(out[ms[0]:].cpu())
        at = [a + m for a, m in zip(at, ms)]
    assert at == total
    pg.k, pg.v = pg.dk.cpu(), pg.dv.cpu()                                     # what the calls wrote, checked on its own first
    q = []
    for b in (0, 1):
        k, v = pg.held(b)
        y, e = paged.turned(x[b][:, nq:nq + nkv], torch.arange(total[b]), f, amp)
        paged.close(k, y, e, "K")
        assert torch.equal(v, x[b][:, nq + nkv:].to(torch.bfloat16))
        q.append(paged.turned(x[b][:, :nq], torch.arange(total[b]), f, amp)[0])
    q = torch.cat(q)
    if dtype == torch.bfloat16:
        q = q.to(dtype)                                                        # a rotated q is rounded to its type
    else:
        q = q.float()
    want, z, eo, ez = paged.attention(pg, q, hd ** -0.5)
    # q itself may be off by the rotation's error, and in bf16 by a step where that crosses a rounding: one more rounding of every score
    eo = eo + (2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -20) * want.abs().amax() * 4
    paged.close(torch.cat([torch.cat(g) for g in got]), want, eo)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("spans,pos0,nq,nkv,hd", [([1] * 700, [(37 * i) % 190 for i in range(700)], 6, 2, 64), ([40] * 100, [(91 * i) % 230 for i in range(100)], 8, 2, 32),
                                                  ([1] * 1024, [i % 3 for i in range(1024)], 2, 1, 32)])
def test_many_sequences_some_with_infinities(spans, pos0, nq, nkv, hd, dtype):
    """Workgroups that take several whole items, and some of an item's tiles: infinities and NaN in V of every ninth sequence."""
    pg = paged.Pages(spans, pos0, nkv, hd, 16, seed=38, fill=float("inf"))
    for b in range(0, len(spans), 9):
        p = pos0[b] // 2
        pg.v[pg.table[pg.slot[b], p // 16], 0, b % hd, p % 16] = (float("inf"), float("nan"), -float("inf"))[b % 3]
    pg.gpu()
    q = torch.randn(pg.rows, nq, hd, generator=pg.gen).to(dtype)
    out, lse = call(pg, q, 0.2)
    check(pg, q, 0.2, 0, out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_long_span_whose_first_pages_are_gone(dtype):
    pg = paged.Pages([150, 33], [300, 70], 2, 128, 32, seed=39).gpu()
    q = torch.randn(pg.rows, 6, 128, generator=pg.gen).to(dtype)
    pg.dtable[pg.slot[0].item(), :7] = -1                                     # positions 0 .. 223; the first row sees 241 .. 300
    flags = torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse = call(pg, q, 0.1, window=60, flags=flags)
    assert flags.tolist() == [0, 0]
    check(pg, q, 0.1, 60, out, lse)
    pg.dtable[pg.slot[0].item(), 8] = 10 ** 9                                 # 256 .. 287: seen
    call(pg, q, 0.1, window=60, flags=flags)
    assert flags.tolist() == [16, 0]


def test_results_repeat_and_do_not_depend_on_the_scratch():
    """Twice the same bits, with different scratch contents, whatever ran before in it."""
    for spans, pos0 in (([1] * 20, [100 * i for i in range(20)]), ([90, 400, 1], [700, 30, 2000])):
        pg = paged.Pages(spans, pos0, 2, 128, 64, seed=40).gpu()
        q = torch.randn(pg.rows, 14, 128, generator=pg.gen).to(torch.bfloat16)
        import paper_2507_17307_amd as P
        n = P.rs_paged_attention_scratch_bytes(pg.cache, pg.n, pg.rows, 14)
        dq, got = q.cuda(), []
        for fill in (0, 255, 127):
            out, lse = torch.empty_like(dq), torch.empty(pg.rows, 14, device="cuda")
            s = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
            P.rs_paged_attention(pg.cache, pg.n, pg.rows, pg.dslot, pg.doff, pg.dpos, dq, 0.09, 0, out, lse, s)
            P.rs_paged_attention(pg.cache, pg.n, pg.rows, pg.dslot, pg.doff, pg.dpos, dq, 0.09, 0, out, lse, s)
            got.append((out.cpu(), lse.cpu()))
        assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_two_calls_at_once_with_scratch_of_their_own():
    import paper_2507_17307_amd as P
    pg = paged.Pages([60, 61], [900, 1000], 2, 128, 64, seed=41).gpu()
    q = torch.randn(pg.rows, 8, 128, generator=pg.gen).to(torch.bfloat16).cuda()
    n = P.rs_paged_attention_scratch_bytes(pg.cache, pg.n, pg.rows, 8)
    want, _ = call(pg, q.cpu(), 0.09)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for _ in range(2)]
    scr = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, c in zip(streams, outs, scr):
            P.rs_paged_attention(pg.cache, pg.n, pg.rows, pg.dslot, pg.doff, pg.dpos, q, 0.09, 0, o, None, c, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o.cpu(), want) for o in outs)
