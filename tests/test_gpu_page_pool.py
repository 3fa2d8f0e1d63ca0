"""rs_pages_reserve, rs_pages_release, rs_pages_fork, rs_pages_copy and rs_pages_compact against plain lists: every entry, count and place equal."""
import random

import pytest
import torch

import beam

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Both:
    """A pool on the GPU and its model."""

    def __init__(self, n_slots, max_pages, n_pages, page, layers=2, heads=2, hd=32, seed=0, contents=True):
        import paper_2507_17307_amd as P
        self.P = P
        g = torch.Generator().manual_seed(seed)
        k = v = None
        if contents:
            k = torch.randn(layers, n_pages, heads, page, hd, generator=g).to(torch.bfloat16)
            v = torch.randn(layers, n_pages, heads, hd, page, generator=g).to(torch.bfloat16)
        self.model = beam.PoolModel(n_slots, max_pages, n_pages, page, k, v)
        self.table = torch.full((n_slots, max_pages), -1, dtype=torch.int32, device="cuda")
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.k, self.v = (None, None) if k is None else (k.cuda(), v.cuda())
        self.pool = P.PagePool(self.table, self.ref, page, self.k, self.v)
        self.scratch = torch.full((P.rs_pages_scratch_bytes(self.pool, 1024),), 255, dtype=torch.uint8, device="cuda")

    def push(self):
        """The model's state to the GPU."""
        self.table.copy_(ints(self.model.table))
        self.ref.copy_(ints(self.model.ref))

    def same(self, what=""):
        torch.cuda.synchronize()
        assert self.table.tolist() == self.model.table, what
        assert self.ref.tolist() == self.model.ref, what
        if self.k is not None:
            assert torch.equal(self.k.cpu(), self.model.k) and torch.equal(self.v.cpu(), self.model.v), what

    def reserve(self, slot, first, end, what=""):
        flags = ints([0] * len(slot))
        self.P.rs_pages_reserve(self.pool, len(slot), ints(slot), None if first is None else ints(first), ints(end), self.scratch, flags)
        want = self.model.reserve(slot, [0] * len(slot) if first is None else first, end)
        assert flags.tolist() == want, what
        return want

    def release(self, slot, first, end, what=""):
        flags = ints([0] * len(slot))
        self.P.rs_pages_release(self.pool, len(slot), ints(slot), None if first is None else ints(first), ints(end), flags)
        want = self.model.release(slot, [0] * len(slot) if first is None else first, end)
        assert flags.tolist() == want, what
        return want

    def fork(self, n_beams, slot, parent, pos, what=""):
        flags, out = ints([0] * len(slot)), ints([-7] * len(slot))
        self.P.rs_pages_fork(self.pool, len(slot) // n_beams, n_beams, ints(slot), ints(parent), ints(pos), out, self.scratch, flags)
        want, want_pos = self.model.fork(n_beams, slot, parent, pos)
        assert flags.tolist() == want, what
        assert out.tolist() == ([-7] * len(slot) if want_pos is None else want_pos), what
        return want

    def compact(self, what=""):
        used = ints([-1])
        self.P.rs_pages_compact(self.pool, used, self.scratch)
        assert used.tolist() == [self.model.compact()], what


@pytest.mark.parametrize("page", [16, 64, 1024])
def test_reserve_and_release_ranges(page):
    b = Both(5, 7, 20, page, contents=False)
    assert b.reserve([0, 3], None, [1, page]) == [0, 0]
    b.same()
    b.reserve([0, 3, 4], [1, page, 0], [page + 1, page, 0])                  # a page more, nothing, nothing
    b.same()
    b.reserve([2, 1], [page * 3, page * 2 - 1], [page * 7, page * 2 + 1])    # not from the start; to the table's end; across a border
    b.same()
    b.release([2, 0], [page * 4 + 1, 0], [page * 7, page - 1])               # whole pages only: two of the three, none
    b.same()
    b.release([0, 1, 2, 3], None, [page * 7] * 4)
    b.same()
    assert not any(b.model.ref)


def test_pages_are_handed_out_lowest_first_and_in_row_order():
    b = Both(4, 4, 12, 16, contents=False)
    b.reserve([2, 0, 1], None, [32, 48, 16])
    b.same()
    assert b.model.table[2][:2] == [0, 1] and b.model.table[0][:3] == [2, 3, 4] and b.model.table[1][0] == 5
    b.release([0], [16], [48])
    b.reserve([3], None, [64])
    b.same()
    assert b.model.table[3] == [3, 4, 6, 7]


def test_rows_that_no_page_is_left_for():
    b = Both(6, 8, 10, 16, contents=False)
    assert b.reserve([0, 1, 2, 3], None, [16 * 4, 16 * 5, 16 * 2, 0]) == [0, 0, 128, 0]
    b.same()
    assert b.reserve([2, 3], None, [16, 16]) == [0, 128]
    b.same()
    assert b.reserve([2, 3, 1], None, [16, 16, 16]) == [0, 128, 0]           # rows that lack nothing
    b.same()


def test_rows_out_of_range_and_slots_named_twice():
    b = Both(4, 4, 12, 16, contents=False)
    assert b.reserve([4, -1, 1, 1, 2, 3, 0], [0, 0, 0, 16, 0, 20, -1], [16, 16, 16, 32, 65, 10, 16]) == [16, 16, 0, 16, 16, 16, 16]
    b.same()
    b.reserve([0, 2], None, [64, 64])
    assert b.release([0, 0, 4, 2, 2**31 - 1, -2**31], [0, 0, 0, 5, 0, 0], [64, 64, 16, 2**31 - 1, 16, 16]) == [0, 16, 16, 16, 16, 16]
    b.same()


def test_entries_that_are_no_pages():
    b = Both(3, 4, 6, 16, contents=False)
    b.model.table = [[99, -5, 2, 6], [1, -1, 2, 2**31 - 1], [-2**31, 3, 0, -1]]
    b.model.ref = [1, 1, 2, 1, 0, 0]
    b.push()
    b.release([1], [0], [64])
    b.same()
    b.reserve([0, 2], None, [64, 17])
    b.same()
    assert b.model.table == [[1, 4, 2, 5], [-1] * 4, [-2**31, 3, 0, -1]]


@pytest.mark.parametrize("n_slots, n_pages, page", [(130, 5000, 16), (1024, 9000, 16), (300, 70000, 32)])
def test_many_rows_and_pages(n_slots, n_pages, page):
    rng = random.Random(n_slots)
    b = Both(n_slots, 40, n_pages, page, contents=False)
    for step in range(4):
        slot = rng.sample(range(n_slots), rng.choice([1, n_slots // 2, n_slots]))
        first = [rng.randrange(0, 39 * page) for _ in slot]
        end = [min(40 * page, f + rng.choice([0, 1, page, rng.randrange(20 * page)])) for f in first]
        b.reserve(slot, first, end)
        b.same(step)
        slot = rng.sample(range(n_slots), n_slots // 3)
        first = [rng.randrange(0, 39 * page) for _ in slot]
        b.release(slot, first, [rng.choice([f, 40 * page, min(40 * page, f + 100)]) for f in first])
        b.same(step)


def forked(page, hd=32, heads=2, layers=2, seed=0, slots=9, n_pages=60):
    return Both(slots, 6, n_pages, page, layers=layers, heads=heads, hd=hd, seed=seed)


@pytest.mark.parametrize("hd, heads", [(32, 1), (64, 3), (128, 2)])
@pytest.mark.parametrize("page, pos", [(16, 1), (16, 15), (16, 16), (16, 17), (32, 40), (64, 63), (64, 200), (128, 129), (1024, 1000)])
def test_one_state_becomes_several(page, pos, hd, heads):
    b = forked(page, hd, heads, layers=3 if page < 1024 else 1, n_pages=60 if page < 1024 else 12)
    b.reserve([5], None, [pos])
    b.fork(4, [5, 1, 8, 3], [0, 0, 0, 0], [pos, 0, 0, 0])
    b.same()
    b.reserve([5, 1, 8, 3], [pos] * 4, [pos + 1] * 4)
    b.same()
    b.fork(4, [5, 1, 8, 3], [2, 2, -1, 1], [pos + 1] * 4)
    b.same()


def test_states_change_places():
    b = forked(16)
    b.reserve([0, 1, 2, 3], None, [40, 33, 16, 5])
    b.fork(4, [0, 1, 2, 3], [1, 0, 3, 2], [40, 33, 16, 5])
    b.same()
    b.fork(4, [0, 1, 2, 3], [3, 0, 1, 2], [33, 40, 5, 16])
    b.same()
    b.fork(1, [0, 1, 2, 3], [0, 0, 0, 0], [16, 33, 40, 5])                   # everyone its own: nothing moves
    b.same()


def test_last_pages_that_others_hold_are_copied():
    b = forked(16)
    b.reserve([0], None, [48])
    b.fork(3, [0, 1, 2], [0, 0, 0], [48, 0, 0])                              # three whole pages, shared
    b.same()
    # taken back into the second page: all three rows write there next, and a slot outside the call holds it too
    assert b.fork(2, [0, 1], [0, 1], [20, 24]) == [0, 0]
    b.same()
    b.fork(1, [2], [0], [30])                                                # nobody else has it now: it stays
    b.same()
    assert b.model.table[2][1] not in (b.model.table[0][1], b.model.table[1][1])


def test_fork_positions_shorter_and_longer_than_what_is_held():
    b = forked(16)
    b.reserve([0, 1], None, [60, 20])
    b.release([0], [0], [16])                                                # evicted: its first entry names no page
    b.fork(2, [0, 1], [0, 0], [50, 20])
    b.same()
    b.fork(2, [0, 1], [1, 0], [96, 70])                                      # positions whose pages were never there
    b.same()
    b.fork(2, [0, 1], [-1, -1], [0, 0])
    b.same()
    assert not any(b.model.ref)


def test_fork_is_refused_as_a_whole():
    b = forked(16, n_pages=8)
    b.reserve([0, 1, 2, 3], None, [20, 20, 20, 20])
    for slot, parent, pos, want in [([0, 1, 1, 3], [0, 0, 0, 0], [20] * 4, [0, 0, 16, 0]), ([0, 1, 9, 3], [0, 0, 0, 2], [20] * 4, [0, 0, 16, 16]),
                                    ([0, 1, 2, 3], [0, 4, 0, 0], [20] * 4, [0, 16, 0, 0]), ([0, 1, 2, 3], [0, 1, 2, 2], [20, 20, 97, 20], [0, 0, 16, 16]),
                                    ([0, 1, 2, 3], [0, 1, 2, 3], [20, -1, 20, 2**31 - 1], [0, 16, 0, 16]), ([-1, 1, 2, 3], [0, 0, 2, 3], [20] * 4, [16, 16, 0, 0])]:
        assert b.fork(4, slot, parent, pos) == want
        b.same()


def test_fork_without_free_pages_changes_nothing():
    b = forked(16, n_pages=6)
    b.reserve([0, 1, 2, 3], None, [20, 20, 16, 16])
    assert b.fork(4, [0, 1, 2, 3], [1, 1, 2, 3], [20, 20, 16, 16]) == [0] * 4            # the pages that row 0 had are free then
    b.same()
    # a whole page, five last ones and row 3's: one more than there are; with one row less they suffice
    assert b.fork(6, [0, 1, 2, 3, 4, 5], [1, 1, 1, 3, 1, 1], [20, 20, 16, 16, 0, 0]) == [128] * 6
    b.same()
    assert b.fork(6, [0, 1, 2, 3, 4, 5], [1, 1, 1, 3, 1, -1], [20, 20, 16, 16, 0, 0]) == [0] * 6
    b.same()


@pytest.mark.parametrize("groups, beams, page, max_pages", [(1, 1, 16, 3), (3, 5, 16, 40), (32, 4, 16, 12), (1, 64, 32, 9), (128, 8, 16, 11), (2, 3, 16, 900)])
def test_forks_and_growth_step_by_step(groups, beams, page, max_pages):
    rng = random.Random(groups * 100 + beams)
    n = groups * beams
    b = Both(n + 3, max_pages, n * 6 + 3 * max_pages * groups, page, layers=1, heads=1, seed=n)
    slot = rng.sample(range(n + 3), n)
    held = [rng.randrange(1, max_pages * page - 40) for _ in range(groups)]
    pos = [held[r // beams] if r % beams == 0 else 0 for r in range(n)]
    b.reserve(slot, None, pos)
    b.fork(beams, slot, [0] * n, pos)
    b.same()
    pos = [held[r // beams] for r in range(n)]
    for step in range(3):
        grow = rng.choice([1, 1, 13])
        b.reserve(slot, pos, [p + grow for p in pos])
        pos = [p + grow for p in pos]
        parent = [rng.randrange(beams) for _ in range(n)]
        assert not any(b.fork(beams, slot, parent, pos))
        b.same(step)


def test_copies_within_a_pool_and_between_two():
    import paper_2507_17307_amd as P
    a, b = Both(1, 1, 9, 32, layers=3, heads=2, hd=64, seed=1), Both(1, 1, 40, 32, layers=3, heads=2, hd=64, seed=2)
    P.rs_pages_copy(b.pool, a.pool, 4, ints([0, 8, 3, 3]), ints([39, 0, 5, 6]))
    for s, d in ((0, 39), (8, 0), (3, 5), (3, 6)):
        b.model.k[:, d], b.model.v[:, d] = a.model.k[:, s], a.model.v[:, s]
    b.same()
    a.same()
    flags = ints([0] * 6)
    P.rs_pages_copy(a.pool, b.pool, 6, ints([39, 40, -1, 20, 21, 2**31 - 1]), ints([1, 2, 3, 9, 4, 5]), flags)
    for s, d in ((39, 1), (21, 4)):
        a.model.k[:, d], a.model.v[:, d] = b.model.k[:, s], b.model.v[:, s]
    a.same()
    assert flags.tolist() == [0, 16, 16, 16, 0, 16]
    P.rs_pages_copy(a.pool, a.pool, 3, ints([1, 6, 2]), ints([0, 6, 8]))
    for s, d in ((1, 0), (2, 8)):
        a.model.k[:, d], a.model.v[:, d] = a.model.k[:, s], a.model.v[:, s]
    a.same()


@pytest.mark.parametrize("page, hd, heads, layers", [(16, 32, 1, 1), (16, 128, 3, 2), (256, 64, 5, 1), (1024, 128, 2, 1), (64, 128, 8, 3)])
def test_copies_of_all_page_sizes(page, hd, heads, layers):
    import paper_2507_17307_amd as P
    b = Both(1, 1, 7, page, layers, heads, hd, seed=3)
    P.rs_pages_copy(b.pool, b.pool, 2, ints([6, 1]), ints([0, 3]))
    for s, d in ((6, 0), (1, 3)):
        b.model.k[:, d], b.model.v[:, d] = b.model.k[:, s], b.model.v[:, s]
    b.same()


@pytest.mark.parametrize("n_pages, used", [(1, 0), (1, 1), (2, 1), (65, 30), (1024, 1024), (1025, 600), (5000, 2500), (3000, 0), (4097, 4096)])
def test_compaction(n_pages, used):
    rng = random.Random(n_pages + used)
    b = Both(8, 700, n_pages, 16, layers=1, heads=1, seed=n_pages)
    held = rng.sample(range(n_pages), used)
    for i, p in enumerate(held):
        b.model.table[i % 8][i // 8] = p
        b.model.ref[p] += 1
        if i % 5 == 0:
            b.model.table[(i + 1) % 8][699 - i // 8] = p
            b.model.ref[p] += 1
    b.model.table[3][650] = n_pages                                          # (no page: it stays)
    b.push()
    b.compact()
    b.same()
    assert all(n > 0 for n in b.model.ref[:used]) and not any(b.model.ref[used:])
    b.compact()
    b.same()


def test_a_run_of_calls_replayed():
    """Reserve, fork, release and compact in one captured graph, replayed on changing slots and parents."""
    import paper_2507_17307_amd as P
    b = Both(6, 8, 50, 16, layers=2, heads=2, seed=9)
    slot, parent, pos, end, used = ints([0, 1, 2, 3]), ints([0] * 4), ints([21, 0, 0, 0]), ints([22] * 4), ints([0])
    limit = ints([8 * 16] * 4)
    b.reserve([0], None, [21])

    def call():
        P.rs_pages_fork(b.pool, 1, 4, slot, parent, pos, pos, b.scratch)
        P.rs_pages_reserve(b.pool, 4, slot, pos, end, b.scratch)
        P.rs_pages_release(b.pool, 4, slot, end, limit)
        P.rs_pages_compact(b.pool, used, b.scratch)

    def model():
        flags, out = b.model.fork(4, slot.tolist(), parent.tolist(), pos_before)
        assert not any(flags)
        b.model.reserve(slot.tolist(), out, end.tolist())
        b.model.release(slot.tolist(), end.tolist(), limit.tolist())
        return out, b.model.compact()
    pos_before = pos.tolist()
    call()
    out, n = model()
    b.same()
    assert pos.tolist() == out and used.tolist() == [n]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for parents, new_end, move in [([0, 1, 2, 3], 23, [0, 1, 2, 3]), ([2, 2, 1, 0], 31, [0, 1, 2, 3]), ([3, 0, 0, 1], 34, [0, 1, 2, 3]), ([1, 1, 1, 1], 50, [0, 1, 2, 3])]:
        parent.copy_(ints(parents))
        pos_before = [int(e) for e in end.tolist()]
        pos.copy_(end)
        end.copy_(ints([new_end] * 4))
        graph.replay()
        out, n = model()
        b.same(parents)
        assert pos.tolist() == out and used.tolist() == [n]


def test_another_stream_than_the_current_one():
    b = Both(4, 8, 40, 16, seed=12)
    stream = torch.cuda.Stream()
    slot, parent, pos = ints([0, 1, 2]), ints([0, 0, 0]), ints([21, 0, 0])
    torch.cuda.synchronize()
    b.P.rs_pages_reserve(b.pool, 1, slot, None, pos, b.scratch, stream=stream)
    b.P.rs_pages_fork(b.pool, 1, 3, slot, parent, pos, pos, b.scratch, stream=stream)
    stream.synchronize()
    b.model.reserve([0], [0], [21])
    b.model.fork(3, [0, 1, 2], [0, 0, 0], [21, 0, 0])
    b.same()


def test_pages_beyond_two_gigabytes():
    """A pool whose K has more than 2^31 bytes and 2^31 elements: the last pages go and come."""
    import paper_2507_17307_amd as P
    n_pages, page, hd, heads = 1100, 1024, 128, 16
    k = torch.zeros(1, n_pages, heads, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(1, n_pages, heads, hd, page, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2 ** 31
    table, ref = torch.full((2, 2), -1, dtype=torch.int32, device="cuda"), torch.ones(n_pages, dtype=torch.int32, device="cuda")
    pool = P.PagePool(table, ref, page, k, v)
    for t in (k, v):
        t[0, n_pages - 1] = torch.randn(t.shape[2:], device="cuda").to(torch.bfloat16)
    P.rs_pages_copy(pool, pool, 2, ints([n_pages - 1, n_pages - 1]), ints([0, n_pages - 2]))
    torch.cuda.synchronize()
    for t in (k, v):
        assert torch.equal(t[0, 0], t[0, n_pages - 1]) and torch.equal(t[0, n_pages - 2], t[0, n_pages - 1]) and bool(t[0, 0].any())
        assert not t[0, 1:n_pages - 2].any()
