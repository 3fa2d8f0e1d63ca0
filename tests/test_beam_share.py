"""What each wave of k_beam_scan takes of a row (beam_share in csrc/beam_plan.h): every value once, whatever the row's address, length and type.  No GPU needed."""
import ctypes as C
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_17307_amd", "csrc")
WRAP = """
#include "beam_plan.h"
using namespace rs;
extern "C" int waves() { return BEAM_WAVES; }
extern "C" int batch() { return BEAM_BATCH; }
extern "C" void share(int address, int bytes, int vocab, int parts, int part, int wave, int *out) {
    const BeamShare s = beam_share(address % 16, bytes, vocab, parts, part, wave);
    out[0] = s.before; out[1] = s.unit_0; out[2] = s.unit_end; out[3] = s.ends;
}
// how often each value is taken by the workgroups of a row; the values a lane would take beyond a wave's 64 ends are counted as errors
extern "C" int count(int address, int bytes, int vocab, int parts, unsigned char *times) {
    int wrong = 0;
    for (int part = 0; part < parts; ++part)
        for (int wave = 0; wave < BEAM_WAVES; ++wave) {
            const BeamShare s = beam_share(address % 16, bytes, vocab, parts, part, wave);
            const int unit = 16 / bytes;
            if (s.unit_end > s.unit_0) wrong += (address + s.before * bytes) % 16 != 0;
            wrong += s.ends < 0 || s.ends > 64 || s.unit_0 < 0;
            for (long long i = s.before + (long long)s.unit_0 * unit; i < s.before + (long long)s.unit_end * unit; ++i) if (i < 0 || i >= vocab) ++wrong; else ++times[i];
            for (int i = 0; i < s.ends; ++i) { const int t = beam_end_token(s, i); if (t < 0 || t >= vocab) ++wrong; else ++times[t]; }
        }
    return wrong;
}
extern "C" int parts_of(int rows, int beams, int vocab, int n_out) { return beam_plan(rows, beams, vocab, n_out, 1024).parts; }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("beam_share")
    src, so = d / "wrap.cpp", d / "libbeam_share.so"
    src.write_text(WRAP)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", CSRC, str(src), "-o", str(so)], check=True)
    return C.CDLL(str(so))


def every_value_once(plan, address, size, vocab, parts):
    times = (C.c_ubyte * vocab)()
    assert plan.count(address, size, vocab, parts, times) == 0
    assert bytes(times) == b"\x01" * vocab, (address, size, vocab, parts)


@pytest.mark.parametrize("size", [2, 4])
def test_short_rows_at_every_address(plan, size):
    for address in range(0, 16, size):
        for vocab in list(range(1, 40)) + [63, 64, 65, 255, 1023, 1024, 1025, 1039]:
            for parts in (1, 2, 5, 64):
                every_value_once(plan, address, size, vocab, parts)


@pytest.mark.parametrize("size", [2, 4])
def test_rows_of_all_lengths_in_their_plans_parts(plan, size):
    rng = random.Random(size)
    for _ in range(300):
        beams, n_out = rng.choice([1, 4, 16, 64]), rng.choice([1, 4, 32, 64])
        vocab = rng.choice([4095, 4096, 4097, 16387, 50257, 152064, rng.randint(1000, 160000)])
        every_value_once(plan, rng.randrange(0, 16, size), size, vocab, plan.parts_of(beams * rng.choice([1, 8, 128]), beams, vocab, n_out))


@pytest.mark.parametrize("size", [2, 4])
@pytest.mark.parametrize("vocab", [2**31 - 1, 2**31 - 8, 2**30 + 5])
@pytest.mark.parametrize("parts", [1, 7, 64])
def test_the_longest_rows(plan, size, vocab, parts):
    """The waves' pieces lie one behind the other, and with the single values they are the row (no number overflows: the wrapper checks)."""
    unit, step = 16 // size, plan.waves()
    for address in (0, size, 16 - size):
        out, at, ends = (C.c_int * 4)(), 0, 0
        for part in range(parts):
            for wave in range(step):
                plan.share(address, size, vocab, parts, part, wave, out)
                assert out[1] == at and out[2] >= at
                at, ends = out[2], ends + out[3]
        assert out[0] == (16 - address) % 16 // size and at * unit + ends == vocab and ends - out[0] < unit


def test_every_wave_that_has_pieces_can_have_a_border(plan):
    """Sharing by as many waves as the pieces fill leaves each of those at least half a batch."""
    out = (C.c_int * 4)()
    for vocab in (1025, 4097, 8200, 50257, 152064):
        for parts in (1, 5, 38):
            held = []
            for part in range(parts):
                for wave in range(plan.waves()):
                    plan.share(0, 4, vocab, parts, part, wave, out)
                    held.append(4 * (out[2] - out[1]))
            held = [h for h in held if h]
            assert max(held) - held[0] == 0 and (len(held) == 1 or min(held[:-1]) >= plan.batch() // 2)
