"""Calls of rs_beam_select with double scores that are refused before anything is launched: no GPU needed."""
import pytest
import torch

from test_beam_args import select

F64 = 256


@pytest.mark.parametrize("change, status, word", [
    (dict(dtype=F64 + 2), -1, "dtype"), (dict(dtype=2 * F64), -1, "dtype"), (dict(dtype=3 * F64), -1, "dtype"), (dict(dtype=-F64), -1, "dtype"), (dict(dtype=F64 - 2**31), -1, "dtype"),
    (dict(dtype=F64, score=4100), -1, "8-byte"), (dict(dtype=F64 + 1, score_out=4100), -1, "8-byte"), (dict(dtype=F64, score=4098), -1, "4-byte"),
    (dict(dtype=F64 + 1, logits=4097), -1, "aligned"), (dict(dtype=F64, bytes=16), -1, "smaller"), (dict(dtype=F64, score=None), -1, "null"),
])
def test_select_refuses(change, status, word):
    import paper_2507_17307_amd as P
    assert P.RS_SCORES_F64 == F64
    assert select(P.lib, **change) == status and word in P.rs_last_error(), P.rs_last_error()


def test_binding_refuses_scores_of_two_types():
    import paper_2507_17307_amd as P
    x, ints, scratch = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    for score, out in ((x[0].double(), x[0]), (x[0], x[0].double()), (x[0].half(), x[0].half()), (x[0].double()[:3], x[0].double()), (x[0].double(), x[0].double()[:3]), (x.double()[:, 0], x[0].double())):
        with pytest.raises(ValueError, match="d_score"):
            P.rs_beam_select(x, 2, 2, None, score, None, -1, 0.0, None, 2, ints, ints, out, None, scratch)
    with pytest.raises(ValueError, match="GPU"):                                                 # (all well, but on the CPU)
        P.rs_beam_select(x, 2, 2, None, x[0].double(), None, -1, 0.0, None, 2, ints, ints, x[0].double(), None, scratch)
