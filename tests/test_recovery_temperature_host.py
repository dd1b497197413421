"""Temperatures whose inverse is beyond fp32 are refused: a logit of 0 would give 0 times infinity, a NaN."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def test_temperatures_without_an_inverse(P):
    from paper_2508_02322_b200.binding import camera_distill_t
    lib = P.lib
    for tau in (1e-45, 1e-40, 4e-39):
        d = camera_distill_t(4096, 100, 4, 1, 100, 4096, 4096, 8, tau, 0)
        assert lib.camera_token_logprobs(4096, 1, 100, 4, 100, 4096, 2, C.c_float(tau), 4096, 4096, 4096, 4096, None) == -1
        assert lib.camera_distill_forward(C.byref(d), 4096, None, None, None) == -1
        assert lib.camera_distill_backward(C.byref(d), 4096, 4096, 4096, 8192, 100, None) == -1
        assert lib.camera_distill_step(C.byref(d), 4096, 4096, 8192, 100, None) == -1
    for tau in (1e-37, 1.0, 1e30):                  # these are taken (nothing to do: no rows)
        assert lib.camera_token_logprobs(None, 1, 100, 0, 100, None, 0, C.c_float(tau), None, None, None, None, None) == 0
