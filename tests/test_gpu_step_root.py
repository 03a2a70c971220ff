"""The square root of the 8-bit step: r = sqrt(v) is kept in a state, so it is the correctly rounded one, checked for every number
that the short form is used for."""
import ctypes as C
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LIB = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "libroot_check.so")
LIMIT = 0x53800000                       # the bits of 2^40


@pytest.fixture(scope="module")
def check():
    lib = C.CDLL(LIB)                    # built by __graft_entry__.build()
    lib.root_check.restype, lib.root_check.argtypes = C.c_int32, [C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p]

    def run(first, count):
        out = torch.tensor([0, 0x7fffffff], dtype=torch.int32, device="cuda")
        assert lib.root_check(first, count, out.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        return out.tolist()
    return run


def test_every_root_below_2_to_the_40_is_correctly_rounded(check):
    """Zero, the subnormal numbers, and all others up to the last below 2^40: 1.4 G numbers."""
    step = 1 << 28
    for first in range(0, LIMIT, step):
        wrong, lowest = check(first, min(step, LIMIT - first))
        assert wrong == 0, f"{wrong} roots of the numbers from {first:#x} on differ, the first that of {lowest:#x}"


def test_the_comparison_sees_a_root_that_is_not_right(check):
    """What lies beyond the form's range is scaled out of float32: infinite there, and counted."""
    wrong, lowest = check(0x7f000000, 1 << 20)                  # from 2^127 on
    assert wrong > 0 and lowest >= 0x7f000000
