"""Gradients of logits never go on top of the logits: refused before anything is launched (no kernel runs in this file)."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1708_02983_amd", "libeasgd_hip.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libeasgd_hip.so not built (run __graft_entry__.build())")

AT, TEACHER = 0x100000, 0x10000        # never dereferenced: every call below has to be refused


@pytest.mark.parametrize("dtype, size", [(0, 4), (1, 2), (2, 2)])
@pytest.mark.parametrize("rows, V, ld, dld, shift", [
    (5, 100, 100, 100, 0),             # in place
    (5, 100, 128, 128, 0), (1, 5000, 5000, 5000, 0), (300, 5000, 5000, 5000, 0),
    (5, 100, 100, 100, 1), (5, 100, 100, 100, -1), (5, 100, 100, 100, 300), (5, 100, 100, 100, -300),      # other rows' memory
    (5, 100, 150, 150, 99), (5, 100, 150, 150, 51), (5, 100, 150, 150, -99), (5, 100, 150, 150, 4 * 150 + 99),
    (1, 100, 1000, 2000, 99), (1, 100, 1000, 2000, -99),
    (5, 100, 400, 500, 150), (5, 100, 500, 400, 0),                                                        # two strides in one range
])
def test_refused(dtype, size, rows, V, ld, dld, shift):
    import paper_1708_02983_amd as hip
    lib = hip.lib()
    out = AT + shift * size
    teacher = (TEACHER, TEACHER, None, 3, None, 1.0, 0.0)
    assert lib.easgd_distill(AT, dtype, rows, V, ld, *teacher, 1.0, TEACHER, out, dld, TEACHER, 1 << 40, None) == -1
    assert lib.easgd_last_error() == b"easgd_distill: dlogits must not overlap logits"
    assert lib.easgd_distill_grad(AT, dtype, rows, V, ld, *teacher, TEACHER, None, 1.0, out, dld, None) == -1
    assert lib.easgd_last_error() == b"easgd_distill_grad: dlogits must not overlap logits"
