"""How a row is dealt to workgroups (csrc/beam_plan.h), and what the compiler says of the kernels of beam search: no GPU needed."""
import ctypes as C
import os
import random
import subprocess

import pytest

from test_no_spills import needs_tools, spills

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_17307_amd", "csrc")
WRAP = """
#include "beam_plan.h"
extern "C" int plan(int rows, int beams, int vocab, int n_out, int slots, int *out) {
    const rs::BeamPlan p = rs::beam_plan(rows, beams, vocab, n_out, slots);
    out[0] = p.parts; out[1] = p.batches;
    return rs::BEAM_WAVES * rs::BEAM_BATCH;
}
extern "C" int limits(int *out) { out[0] = rs::BEAM_PARTS; out[1] = rs::BEAM_KEYS; out[2] = rs::BEAM_MAX; return 0; }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("beam_plan")
    src, so = d / "wrap.cpp", d / "libbeam_plan.so"
    src.write_text(WRAP)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    return C.CDLL(str(so))


def test_every_plan_covers_the_row_and_keeps_the_limits(plan):
    out, limit = (C.c_int * 2)(), (C.c_int * 3)()
    plan.limits(limit)
    parts_most, keys_most, beam_max = limit
    assert keys_most >= beam_max * beam_max                                   # (a part at least, whatever the beams and candidates)
    rng = random.Random(3)
    for _ in range(3000):
        beams, n_out = rng.choice([1, 2, 4, 8, 31, 64, rng.randint(1, 64)]), rng.choice([1, 4, 32, 64, rng.randint(1, 64)])
        rows = beams * rng.choice([1, 2, 10, 128, rng.randint(1, 65535 // beams)])
        vocab = rng.choice([1, 4095, 4096, 4097, 152064, 2**31 - 1, rng.randint(1, 300000)])
        step = plan.plan(rows, beams, vocab, n_out, 1024, out)
        parts, batches = out
        assert 1 <= parts <= parts_most and parts * beams * n_out <= keys_most and batches >= 1
        assert parts * batches * step >= vocab and (parts - 1) * batches * step < vocab


@pytest.mark.parametrize("rows, beams, n_out, parts, batches", [(4, 4, 4, 38, 1), (128, 4, 4, 8, 5), (384, 16, 32, 5, 8), (64, 64, 64, 1, 38)])
def test_plans_of_one_vocabulary(plan, rows, beams, n_out, parts, batches):
    out = (C.c_int * 2)()
    plan.plan(rows, beams, 152064, n_out, 1024, out)
    assert list(out) == [parts, batches]


@needs_tools
def test_beam_search_kernels_do_not_spill(tmp_path):
    kernels = {n: s for n, s in spills(tmp_path).items() if "k_beam_" in n or "k_pool_" in n}
    assert len(kernels) == 3 + 6 and not any(kernels.values()), kernels       # scan of two types, join; release, reserve, copy, compact, fork of two sizes
