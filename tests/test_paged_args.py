"""Calls on caches in pages that are refused, and the host arithmetic behind them (csrc/paged_plan.h, rs_rope_frequencies): no GPU needed."""
import ctypes as C
import math
import os
import random
import subprocess

import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_17307_amd", "csrc")
WRAP = """
#include "paged_plan.h"
extern "C" int span(const int *slot, const int *off, const int *pos0, int n_seqs, int n_rows, int n_slots, int max_pages, int shift, int b, rs::Span *s) {
    rs::PagedSpans a{slot, off, pos0, nullptr, nullptr, n_seqs, n_rows, n_slots, 1, max_pages, shift, 1, nullptr};
    return rs::paged_span(a, b, *s);
}
extern "C" int info_span(const int *info, int n_rows, int n_slots, int max_pages, int shift, int b, rs::Span *s) {
    rs::PagedSpans a{nullptr, nullptr, nullptr, nullptr, info, 1, n_rows, n_slots, 1, max_pages, shift, 1, nullptr};
    return rs::paged_span(a, b, *s);
}
extern "C" int n_blocks(int m, int rows) { return rs::paged_blocks(rs::Span{0, m, 0, 0}, rows); }
extern "C" void tiles(int m, int p0, int rows, int window, int j, int *t) { rs::paged_tiles(rs::Span{0, m, 0, p0}, rows, window, 6, j, t[0], t[1]); }
extern "C" long long run(long long T, int W, int w) { return rs::paged_run(T, W, w); }
extern "C" int run_of(long long T, int W, long long t) { return rs::paged_run_of(T, W, t); }
extern "C" int blocks(int m, int p0) { return rs::append_blocks_of(rs::Span{0, m, 0, p0}); }
extern "C" int blocks_most(int n_seqs, int n_rows) { return rs::append_blocks_most(n_seqs, n_rows); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_plan")
    src, so = d / "wrap.cpp", d / "libpaged_plan.so"
    src.write_text(WRAP)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.run.restype, lib.run.argtypes, lib.run_of.argtypes = C.c_longlong, [C.c_longlong, C.c_int, C.c_int], [C.c_longlong, C.c_int, C.c_longlong]
    return lib


def ints(*v):
    return (C.c_int * len(v))(*v)


def test_spans_out_of_range_are_told(plan):
    s = (C.c_int * 4)()

    def span(slot, off, pos0, b=0, n_rows=10, n_slots=4, max_pages=3, shift=4):
        return plan.span(ints(*slot), None if off is None else ints(*off), ints(*pos0), len(slot), n_rows, n_slots, max_pages, shift, b, s)

    assert span([3], [0, 5], [43]) and list(s) == [0, 5, 3, 43]            # the last position a slot has
    assert not span([3], [0, 5], [44])
    assert span([0], [4, 4], [48]) and not span([0], [4, 4], [49])         # an empty span at the end of a slot
    assert not span([0], [0, 5], [-1]) and not span([-1], [0, 5], [0]) and not span([4], [0, 5], [0])
    assert not span([0], [0, 11], [0]) and not span([0], [-1, 5], [0]) and not span([0], [5, 4], [0])
    assert not span([0], [0, 5], [2**31 - 1])                              # no overflow in the sum
    assert not span([0], [-2**31, 2**31 - 1], [0])
    assert span([0, 1], None, [0, 7], b=1) and list(s) == [1, 1, 1, 7]
    assert span([0], [0, 5], [2**30 - 5], max_pages=2**26) and not span([0], [0, 5], [2**30 - 4], max_pages=2**26)


def test_spans_of_a_prepared_row_table(plan):
    s = (C.c_int * 4)()
    table = ints(3, 8, 2, 10, -1, 0, 0, 0, 0, 4, 9, 0)
    assert plan.info_span(table, 10, 4, 3, 4, 0, s) and list(s) == [3, 5, 2, 10]
    assert not plan.info_span(table, 10, 4, 3, 4, 1, s) and not plan.info_span(table, 10, 4, 3, 4, 2, s)


def test_tiles_of_a_block_are_those_that_its_rows_see(plan):
    rng, t = random.Random(2), (C.c_int * 2)()
    for _ in range(3000):
        m, p0, rows, window = rng.randint(1, 300), rng.choice([0, 1, 63, 64, rng.randint(0, 5000)]), rng.choice([1, 2, 5, 18, 25, 128]), rng.choice([0, 0, 1, 63, 64, 65, 1000, 2**31 - 1])
        j = rng.randrange(plan.n_blocks(m, rows))
        seen = [x for r in range(j * rows, min(m, (j + 1) * rows)) for x in (max(0, p0 + r - window + 1) if window else 0, p0 + r)]
        plan.tiles(m, p0, rows, window, j, t)
        assert (t[0], t[1]) == (min(seen) // 64, max(seen) // 64 + 1)
    assert plan.n_blocks(0, 5) == 0 and plan.n_blocks(11, 5) == 3


@pytest.mark.parametrize("T", [1, 7, 511, 512, 513, 100003, 2**31 - 1, 2**31, 2**40 + 12345])
@pytest.mark.parametrize("W", [1, 8, 256, 512, 1024])
def test_runs_share_the_tiles_evenly(plan, T, W):
    W = min(W, T)
    starts = [plan.run(T, W, w) for w in range(W + 1)]
    assert starts[0] == 0 and starts[-1] == T
    sizes = {b - a for a, b in zip(starts, starts[1:])}
    assert max(sizes) - min(sizes) <= 1 and min(sizes) >= 1
    for t in {0, T - 1, T // 2, T // 3} | {s for s in starts[1:-1][::37]} | {s - 1 for s in starts[1:][::41]}:
        w = plan.run_of(T, W, t)
        assert starts[w] <= t < starts[w + 1]


def test_append_launches_a_workgroup_for_every_block_of_positions(plan):
    rng = random.Random(1)
    for _ in range(2000):
        n = rng.randint(1, 20)
        m = [rng.choice([0, 1, 1, 2, rng.randint(1, 400)]) for _ in range(n)]
        p = [rng.randint(0, 1000) for _ in range(n)]
        need = sum(len({(p0 + i) // 64 for i in range(k)}) for k, p0 in zip(m, p))
        assert sum(plan.blocks(k, p0) for k, p0 in zip(m, p)) == need
        assert sum(m) < 1 or need <= plan.blocks_most(n, sum(m) + rng.randint(0, 3))


def test_frequencies_follow_their_definitions():
    import paper_2507_17307_amd as P
    f, amp = P.rs_rope_frequencies(128, 1e6)
    want = 1e6 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)
    assert amp == 1.0 and torch.allclose(f, want, rtol=1e-14, atol=0)
    f, amp = P.rs_rope_frequencies(64, 1e4, P.ROPE_LINEAR, 8.0)
    assert amp == 1.0 and torch.allclose(f, 1e4 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64) / 8, rtol=1e-14, atol=0)
    f, amp = P.rs_rope_frequencies(128, 1e6, P.ROPE_BY_PARTS, 4.0, original_ctx=32768)
    assert abs(amp - (0.1 * math.log(4.0) + 1)) <= 2.0 ** -24 * amp
    turns = 32768 * want / (2 * math.pi)                      # wavelengths that fit the original context
    assert torch.allclose(f[turns >= 32], want[turns >= 32], rtol=1e-14, atol=0) and torch.allclose(f[turns <= 1], want[turns <= 1] / 4, rtol=1e-14, atol=0)
    mid = (turns > 1) & (turns < 32)
    keep = (turns - 1) / 31
    assert mid.any() and torch.allclose(f[mid], (want * (keep + (1 - keep) / 4))[mid], rtol=1e-14, atol=0)


@pytest.mark.parametrize("args", [(0, 1e6), (7, 1e6), (64, 1.0), (64, float("inf")), (64, 1e6, 3), (64, 1e6, 1, 0.5), (64, 1e6, 2, 2.0, 0.5), (64, 1e6, 2, 2.0, 32768.0, 1.0, 1.0),
                                  (64, 1e6, 2, float("nan"))])
def test_frequencies_refuse(args):
    import paper_2507_17307_amd as P
    with pytest.raises(P.RsError) as e:
        P.rs_rope_frequencies(*args)
    assert e.value.status == -1


def cache(P, **kw):
    v = dict(k=256, v=256, page_table=4, n_pages=9, page_size=16, n_slots=2, max_pages=4, n_kv_heads=2, head_dim=64)
    v.update(kw)
    return P.binding._RsPagedKv(*v.values())


BAD_CACHES = [dict(page_table=6), dict(k=None), dict(v=None), dict(page_table=None), dict(k=8), dict(v=264), dict(n_pages=0), dict(page_size=8), dict(page_size=48), dict(page_size=2048),
              dict(n_slots=0), dict(max_pages=0), dict(page_size=16, max_pages=2**26 + 1), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(head_dim=96), dict(head_dim=0)]


def attention(P, c, n_seqs=1, n_rows=4, slot=4, off=4, pos0=4, dtype=0, n_q=4, q=16, qs=256, scale=0.1, window=0, out=512, outs=256, scratch=256, size=1 << 40):
    return P.lib.rs_paged_attention(c if c is None else C.byref(c), n_seqs, n_rows, slot, off, pos0, dtype, n_q, q, qs, scale, window, out, outs, None, None, scratch, size, None)


def append(P, c, n_seqs=1, n_rows=4, slot=4, off=4, pos0=4, rope=None, dtype=0, n_q=4, q=16, qs=256, k=16, ks=256, v=16, vs=256, out=512, outs=256):
    return P.lib.rs_paged_append(c if c is None else C.byref(c), n_seqs, n_rows, slot, off, pos0, None if rope is None else C.byref(rope), dtype, n_q, q, qs, k, ks, v, vs, out, outs,
                                 None, None)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_malformed_caches_are_refused_before_any_launch(bad):
    import paper_2507_17307_amd as P
    c = cache(P, **bad)
    assert attention(P, c) == -1 and P.rs_last_error()
    assert bad == dict(n_kv_heads=3) or append(P, c) == -1
    assert P.lib.rs_paged_attention_scratch_bytes(C.byref(c), 1, 4, 4) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(n_seqs=0), -1), (dict(n_rows=0), -1), (dict(n_seqs=1025), -2), (dict(n_rows=2**22 + 1), -2), (dict(slot=None), -1), (dict(pos0=None), -1),
    (dict(n_seqs=5, off=None), -1), (dict(dtype=2), -1), (dict(n_q=0), -1), (dict(q=None), -1), (dict(q=8), -1), (dict(qs=252, dtype=1), -1), (dict(qs=192), -1),
    (dict(slot=6), -1), (dict(off=5), -1), (dict(pos0=7), -1), (dict(out=None), -1), (dict(out=520), -1), (dict(outs=255), -1), (dict(outs=128), -1)])
def test_malformed_rows_are_refused_before_any_launch(bad, status):
    import paper_2507_17307_amd as P
    assert attention(P, cache(P), **bad) == status and append(P, cache(P), **bad) == status


@pytest.mark.parametrize("bad", [dict(n_q=5), dict(n_q=34, qs=4096, outs=4096), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(window=-1),
                                 dict(out=16), dict(scratch=None), dict(scratch=128), dict(size=0)])
def test_malformed_attention_arguments_are_refused(bad):
    import paper_2507_17307_amd as P
    assert attention(P, cache(P), **bad) == -1 and P.rs_last_error()
    assert attention(P, None) == -1


def test_malformed_append_and_rope_arguments_are_refused():
    import paper_2507_17307_amd as P
    R = P.binding._RsRope
    for bad in (dict(k=None), dict(k=24), dict(ks=64), dict(v=None), dict(vs=130), dict(q=512, qs=260)):
        assert append(P, cache(P), **bad) == -1, bad
    assert append(P, None) == -1
    ropes = [R(0, 0, 8, 1.0), R(12, 0, 8, 1.0), R(72, 0, 8, 1.0), R(64, 2, 8, 1.0), R(64, 0, None, 1.0), R(64, 0, 4, 1.0), R(64, 0, 8, float("nan"))]
    for r in ropes:
        assert append(P, cache(P), rope=r) == -1

    def rows(rope=R(64, 0, 8, 1.0), n=4, pos=4, dtype=0, heads=2, hd=64, x=16, xs=128, inverse=0, out=512, outs=128):
        return P.lib.rs_rope_rows(None if rope is None else C.byref(rope), n, pos, dtype, heads, hd, x, xs, inverse, out, outs, None)
    for r in ropes + [None]:
        assert rows(rope=r) == -1
    for bad in (dict(n=0), dict(pos=None), dict(dtype=3), dict(heads=0), dict(hd=60), dict(hd=2048, xs=4096, outs=4096), dict(x=None), dict(x=4), dict(xs=126), dict(xs=64),
                dict(inverse=2), dict(out=None), dict(outs=127), dict(x=512, xs=256)):
        assert rows(**bad) == -1, bad
    assert rows(n=2**22 + 1) == -2


def test_the_binding_refuses_tensors_that_do_not_fit():
    import paper_2507_17307_amd as P
    k, v, t = torch.zeros(3, 2, 16, 32, dtype=torch.bfloat16), torch.zeros(3, 2, 32, 16, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32)
    c = P.PagedCache(k, v, t)
    assert (c.n_kv_heads, c.page_size, c.head_dim) == (2, 16, 32)
    for bad in ((k.float(), v, t), (k, k, t), (k, v, t.long()), (k, v, t[0]), (k.transpose(0, 1), v, t), (k, v, torch.zeros(2, 4, dtype=torch.int32)[:, :2])):
        with pytest.raises(ValueError):
            P.PagedCache(*bad)
    with pytest.raises(ValueError):
        P.Rope(torch.zeros(16))
    one, q = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, 32)
    s = torch.zeros(256, dtype=torch.uint8)

    def att(c=c, slot=one, pos=one, q=q, out=q.clone(), lse=None, scratch=s, n=2):
        P.rs_paged_attention(c, 2, n, slot, None, pos, q, 0.1, 0, out, lse, scratch)
    with pytest.raises(ValueError, match="GPU"):                                   # everything fits but the device
        att()
    for bad in (dict(slot=one.long()), dict(slot=one[:1]), dict(pos=one[:1]), dict(q=q.half(), out=q.half()), dict(out=q.bfloat16()), dict(q=q[:, :, :16]), dict(n=3),
                dict(q=torch.zeros(2, 32, 4).transpose(1, 2)), dict(lse=torch.zeros(2, 3)), dict(scratch=None)):
        with pytest.raises(ValueError):
            att(**bad)
    r = P.Rope(torch.zeros(16, dtype=torch.float64))
    for bad in ((r, one, q.half(), q.half()), (r, one, q, q.bfloat16()), (r, one[:1], q, q), (r, one, q, q[:, :2])):
        with pytest.raises(ValueError):
            P.rs_rope_rows(*bad)


@pytest.mark.parametrize("n_pages,page_size", [(0, 64), (-1, 64), (4, 0), (4, -16)])
def test_an_empty_pool_is_refused_before_anything_is_allocated(n_pages, page_size):
    import paper_2507_17307_amd as P
    with pytest.raises(P.RsError) as e:
        P.PagedModel(None, 128, n_pages, page_size)
    assert e.value.status == -1
