"""Scales of an attention's scores that its kernel cannot hold, as a factor times log2(e) in float32."""
import ctypes as C

import numpy as np
import pytest

import test_pages_cpu as T

asr = pytest.importorskip("paper_2603_11273_amd.asr")

BORDER = 2.0 ** 128 / np.log2(np.e)                 # 2.359e38


@pytest.mark.parametrize("scale", [3.0e38, -3.0e38, BORDER * (1 + 2.0 ** -20), 3.4028235e38])
def test_scales_whose_factor_overflows_are_refused(scale):
    assert T.CALLS["attend"](T.attend(scale=scale)) == asr.ASR_EINVAL
    assert T.SIZES["attend"](C.byref(T.attend(scale=scale)), C.byref(C.c_size_t())) == asr.ASR_EINVAL


@pytest.mark.parametrize("scale", [0.0, 1e-38, -0.125, 1e38, BORDER * (1 - 2.0 ** -20)])
def test_scales_that_hold_are_taken(scale):
    assert T.SIZES["attend"](C.byref(T.attend(scale=scale)), C.byref(C.c_size_t())) == asr.ASR_OK
