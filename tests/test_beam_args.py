"""Calls of beam search that are refused before anything is launched: no GPU needed."""
import ctypes as C

import pytest
import torch


def select(lib, **change):
    a = dict(logits=4096, stride=100, dtype=0, groups=2, beams=3, vocab=100, scale=None, score=4096, last=None, eos=-1, penalty=0.0, length=None, n_out=3,
             parent=4096, token=4096, score_out=4096, len_out=None, flags=None, scratch=4096, bytes=1 << 20)
    a.update(change)
    return lib.rs_beam_select(a["logits"], a["stride"], a["dtype"], a["groups"], a["beams"], a["vocab"], a["scale"], a["score"], a["last"], a["eos"], a["penalty"],
                              a["length"], a["n_out"], a["parent"], a["token"], a["score_out"], a["len_out"], a["flags"], a["scratch"], a["bytes"], None)


@pytest.mark.parametrize("change, status, word", [
    (dict(logits=None), -1, "null"), (dict(score=None), -1, "null"), (dict(parent=None), -1, "null"), (dict(scratch=None), -1, "null"),
    (dict(dtype=2), -1, "dtype"), (dict(groups=0), -1, "n_groups"), (dict(beams=0), -1, "n_beams"), (dict(beams=65), -1, "n_beams"),
    (dict(n_out=0), -1, "n_out"), (dict(n_out=65), -1, "n_out"), (dict(vocab=0), -1, "vocab"), (dict(groups=30000), -2, "65535"),
    (dict(stride=99), -1, "row_stride"), (dict(stride=1 << 41), -1, "row_stride"), (dict(eos=100), -1, "eos"), (dict(eos=-2), -1, "eos"),
    (dict(penalty=-0.5), -1, "length_penalty"), (dict(penalty=float("nan")), -1, "length_penalty"), (dict(penalty=float("inf")), -1, "length_penalty"), (dict(penalty=30.5, length=4096), -1, "length_penalty"),
    (dict(penalty=1.0), -1, "lengths"), (dict(len_out=4096), -1, "lengths"), (dict(logits=4098), -1, "aligned"), (dict(logits=4097, dtype=1), -1, "aligned"),
    (dict(token=4098), -1, "4-byte"), (dict(flags=4097), -1, "4-byte"), (dict(scratch=4112), -1, "256-byte"), (dict(bytes=16), -1, "smaller"),
])
def test_select_refuses(change, status, word):
    import paper_2507_17307_amd as P
    assert select(P.lib, **change) == status and word in P.rs_last_error(), P.rs_last_error()


def test_select_scratch():
    import paper_2507_17307_amd as P
    assert P.rs_beam_select_scratch_bytes(1, 1, 1, 1) > 0 and P.rs_beam_select_scratch_bytes(32, 4, 152064, 4) > 0
    for bad in ((0, 1, 10, 1), (1, 0, 10, 1), (1, 65, 10, 1), (1, 1, 0, 1), (1, 1, 10, 0), (1, 1, 10, 65), (2000, 64, 10, 1)):
        assert P.rs_beam_select_scratch_bytes(*bad) == 0


def pool_struct(P, **change):
    a = dict(k=4096, v=4096, page_table=4096, page_ref=4096, n_layers=2, n_pages=8, page_size=16, n_slots=4, max_pages=4, n_kv_heads=2, head_dim=64)
    a.update(change)
    return P.binding._RsPagePool(*a.values())


POOL = [(dict(page_table=None), "null"), (dict(page_ref=None), "null"), (dict(page_table=4097), "aligned"), (dict(page_ref=4098), "aligned"), (dict(n_pages=0), "below 1"),
        (dict(n_slots=0), "below 1"), (dict(max_pages=0), "below 1"), (dict(n_pages=(1 << 30) + 1), "2^30"), (dict(page_size=24), "power"), (dict(page_size=8), "power"),
        (dict(page_size=2048), "power"), (dict(max_pages=1 << 27), "2^30"), (dict(n_slots=1 << 20, max_pages=1 << 20), "2^31")]
CONTENTS = [(dict(k=None), "without pages"), (dict(v=None), "without pages"), (dict(k=4104), "16-byte"), (dict(n_layers=0), "n_layers"), (dict(n_kv_heads=1025), "n_kv_heads"),
            (dict(head_dim=48), "head_dim")]


@pytest.mark.parametrize("change, word", POOL)
def test_every_call_refuses_a_bad_pool(change, word):
    import paper_2507_17307_amd as P
    p, lib, n = C.byref(pool_struct(P, **change)), P.lib, 1 << 20
    good = C.byref(pool_struct(P))
    for status in (lambda: lib.rs_pages_reserve(p, 1, 4096, None, 4096, None, 4096, n, None), lambda: lib.rs_pages_release(p, 1, 4096, None, 4096, None, None),
                   lambda: lib.rs_pages_fork(p, 1, 1, 4096, 4096, 4096, None, None, 4096, n, None), lambda: lib.rs_pages_copy(p, good, 1, 4096, 4096, None, None),
                   lambda: lib.rs_pages_copy(good, p, 1, 4096, 4096, None, None), lambda: lib.rs_pages_compact(p, 4096, 4096, n, None)):
        assert status() == -1 and word in P.rs_last_error(), P.rs_last_error()
    assert lib.rs_pages_scratch_bytes(p, 1) == 0 and lib.rs_pages_scratch_bytes(None, 1) == 0


@pytest.mark.parametrize("change, word", CONTENTS)
def test_calls_that_move_pages_refuse_a_pool_without_them(change, word):
    import paper_2507_17307_amd as P
    p, lib, n = C.byref(pool_struct(P, **change)), P.lib, 1 << 20
    good = C.byref(pool_struct(P))
    for status in (lambda: lib.rs_pages_fork(p, 1, 1, 4096, 4096, 4096, None, None, 4096, n, None), lambda: lib.rs_pages_copy(p, good, 1, 4096, 4096, None, None),
                   lambda: lib.rs_pages_copy(good, p, 1, 4096, 4096, None, None), lambda: lib.rs_pages_compact(p, 4096, 4096, n, None)):
        assert status() == -1 and word in P.rs_last_error(), P.rs_last_error()


def test_a_page_that_no_grid_covers_is_refused_before_anything_is_done():
    import paper_2507_17307_amd as P
    p, lib, n = C.byref(pool_struct(P, n_layers=65536, n_kv_heads=1024, head_dim=128, page_size=1024)), P.lib, 1 << 20
    for call in (lambda: lib.rs_pages_fork(p, 1, 1, 4096, 4096, 4096, None, None, 4096, n, None), lambda: lib.rs_pages_copy(p, p, 1, 4096, 4096, None, None),
                 lambda: lib.rs_pages_compact(p, 4096, 4096, n, None)):
        assert call() == -1 and "too large" in P.rs_last_error(), P.rs_last_error()


def test_rows_and_scratch_of_pool_calls():
    import paper_2507_17307_amd as P
    p, lib, n = C.byref(pool_struct(P)), P.lib, 1 << 20
    for args, status, word in [((0, 4096, None, 4096), -1, "at least one"), ((1025, 4096, None, 4096), -2, "1024"), ((1, None, None, 4096), -1, "null"),
                               ((1, 4096, None, None), -1, "null"), ((1, 4097, None, 4096), -1, "aligned"), ((1, 4096, 4098, 4096), -1, "aligned")]:
        assert lib.rs_pages_reserve(p, *args, None, 4096, n, None) == status and word in P.rs_last_error()
        assert lib.rs_pages_release(p, *args, None, None) == status and word in P.rs_last_error()
    assert lib.rs_pages_reserve(p, 1, 4096, None, 4096, None, None, n, None) == -1 and "256" in P.rs_last_error()
    assert lib.rs_pages_reserve(p, 1, 4096, None, 4096, None, 4096, 16, None) == -1 and "smaller" in P.rs_last_error()
    for args, status, word in [((0, 1, 4096, 4096, 4096), -1, "n_groups"), ((1, 0, 4096, 4096, 4096), -1, "n_beams"), ((512, 3, 4096, 4096, 4096), -2, "1024"),
                               ((1, 1, None, 4096, 4096), -1, "null"), ((1, 1, 4096, None, 4096), -1, "null"), ((1, 1, 4096, 4096, None), -1, "null"),
                               ((1, 1, 4096, 4097, 4096), -1, "aligned")]:
        assert lib.rs_pages_fork(p, *args, None, None, 4096, n, None) == status and word in P.rs_last_error()
    assert lib.rs_pages_fork(p, 1, 1, 4096, 4096, 4096, 4097, None, 4096, n, None) == -1 and "aligned" in P.rs_last_error()
    assert lib.rs_pages_fork(p, 1, 1, 4096, 4096, 4096, None, None, 4352, 16, None) == -1 and "smaller" in P.rs_last_error()
    assert lib.rs_pages_compact(p, None, 4096, n, None) == -1 and lib.rs_pages_compact(p, 4096, 4100, n, None) == -1
    for args, status, word in [((0, 4096, 4096), -1, "pair"), (((1 << 22) + 1, 4096, 4096), -2, "2^22"), ((1, None, 4096), -1, "null"), ((1, 4096, 4098), -1, "aligned")]:
        assert lib.rs_pages_copy(p, p, *args, None, None) == status and word in P.rs_last_error()
    for change in (dict(n_layers=3), dict(page_size=32), dict(n_kv_heads=1), dict(head_dim=32)):
        assert lib.rs_pages_copy(p, C.byref(pool_struct(P, **change)), 1, 4096, 4096, None, None) == -1 and "differ" in P.rs_last_error()
    assert lib.rs_pages_scratch_bytes(p, 0) == 0 and lib.rs_pages_scratch_bytes(p, 1025) == 0 and lib.rs_pages_scratch_bytes(p, 1024) > 1024 * 16


def test_binding_refuses_tensors():
    import paper_2507_17307_amd as P
    table, ref = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)
    k, v = torch.zeros(2, 8, 2, 16, 32, dtype=torch.bfloat16), torch.zeros(2, 8, 2, 32, 16, dtype=torch.bfloat16)
    P.PagePool(table, ref, 16, k, v)
    for args in ((table.long(), ref, 16), (table, ref.float(), 16), (table[0], ref, 16), (table, ref, 16, k, None), (table, ref, 16, k.float(), v.float()), (table, ref, 32, k, v),
                 (table, ref, 16, k, k), (table, ref[:4], 16, k, v), (table.t(), ref, 16), (table, ref, 16, k[0], v[0])):
        with pytest.raises(ValueError):
            P.PagePool(*args)
    pool, ints, x = P.PagePool(table, ref, 16, k, v), torch.zeros(8, dtype=torch.int32), torch.zeros(4, 10)
    out, scratch = torch.zeros(4, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: P.rs_pages_reserve(pool, 9, ints, ints, ints, scratch), lambda: P.rs_pages_release(pool, 1, ints.long(), None, ints),
                 lambda: P.rs_pages_fork(pool, 1, 2, ints[:1], ints, ints, None, scratch), lambda: P.rs_pages_reserve(pool, 1, ints, None, ints, None),
                 lambda: P.rs_pages_copy(pool, pool, 9, ints, ints), lambda: P.rs_pages_compact(pool, ints[:0], scratch),
                 lambda: P.rs_beam_select(x.double(), 2, 2, None, x[0], None, -1, 0.0, None, 2, out, out, x[0], None, scratch),
                 lambda: P.rs_beam_select(x, 3, 2, None, x[0], None, -1, 0.0, None, 2, out, out, x[0], None, scratch),
                 lambda: P.rs_beam_select(x.t(), 2, 2, None, x[0], None, -1, 0.0, None, 2, out, out, x[0], None, scratch),
                 lambda: P.rs_beam_select(x, 2, 2, None, x[0].double(), None, -1, 0.0, None, 2, out, out, x[0], None, scratch),
                 lambda: P.rs_beam_select(x, 2, 2, None, x[0, :3], None, -1, 0.0, None, 2, out, out, x[0], None, scratch),
                 lambda: P.rs_beam_select(x, 2, 2, None, x[0], None, -1, 0.0, None, 3, out, out, x[0], None, scratch),
                 lambda: P.rs_beam_select(x, 2, 2, None, x[0], None, -1, 0.0, None, 2, out, out, x[0], None, None),
                 lambda: P.rs_pages_release(pool, 1, ints, None, ints)):                          # (all well, but on the CPU)
        with pytest.raises(ValueError):
            call()
