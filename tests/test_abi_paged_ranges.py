"""Parameters that kernels take in single precision are refused where that does not hold them (host-side, no GPU)."""
import ctypes

import pytest

from paper_2409_09086_amd import binding as B


@pytest.mark.parametrize("value,ok", [(1e-30, True), (1e30, True), (2.3e38, True), (2.4e38, False), (1e300, False), (1e-38, True), (8e-39, False), (1e-300, False)])
def test_scale(value, ok):
    """scale * log2(e) as a float: neither infinite (every weight would be NaN) nor 0 (so would a hidden one)."""
    L, p = B.lib(), ctypes.c_void_p()
    assert L.infmllm_paged_create(8, 16, 4, 2, 64, B.BF16, ctypes.byref(p)) == B.OK
    assert L.infmllm_paged_set_param(p, B.PAGED_SCALE, value) == (B.OK if ok else B.EINVAL)
    L.infmllm_paged_destroy(p)


@pytest.mark.parametrize("which", [B.ROTARY_MAGNITUDE, B.ROTARY_EPS])
@pytest.mark.parametrize("value,ok", [(1e-30, True), (1e30, True), (3.4e38, True), (3.5e38, False), (1e300, False), (1.2e-38, True), (1e-38, False), (1e-300, False)])
def test_magnitude_and_eps(which, value, ok):
    """An infinite magnitude makes NaN of differences, an eps of 0 beside a row of zeros too."""
    L, r = B.lib(), ctypes.c_void_p()
    assert L.infmllm_rotary_create(64, B.BF16, 100, ctypes.byref(r)) == B.OK
    assert L.infmllm_rotary_set_param(r, which, value) == (B.OK if ok else B.EINVAL)
    L.infmllm_rotary_destroy(r)
