"""Host-only: frequencies that leave the range of a double are refused, and nothing is written."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def K():
    from paper_2606_03458_amd import kvarn
    kvarn.lib()
    return kvarn


@pytest.mark.parametrize("rot,base,kind,factor", [(128, 1e4, "LINEAR", 1e-310), (128, 1e4, "BASE", 1e308), (128, 1e4, "BASE", 5e-324),
                                                 (4, 1e300, "BASE", 1e200), (128, 1e4, "RAMP", 1e-310), (64, 1e4, "BANDS", 1e-310)])
def test_refused(K, rot, base, kind, factor):
    freq, amp = np.full(rot // 2, 7.0), ctypes.c_double(7.0)
    s = K.kvarn_rope_scaling(getattr(K, "KVARN_ROPE_" + kind), factor, 4096.0, 1.0, 32.0)
    st = K.lib().kvarn_rope_frequencies(rot, base, ctypes.byref(s), freq.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), ctypes.byref(amp))
    assert st == -1 and (freq == 7.0).all() and amp.value == 7.0


@pytest.mark.parametrize("kind,factor", [("LINEAR", 1e-290), ("BASE", 1e200), ("BASE", 1e-200), ("RAMP", 1e300), ("BANDS", 1e-200)])
def test_within(K, kind, factor):
    f, amp = K.kvarn_rope_frequencies(128, 1e4, K.kvarn_rope_scaling(getattr(K, "KVARN_ROPE_" + kind), factor, 4096.0, 1.0, 32.0))
    assert np.isfinite(f.numpy()).all() and np.isfinite(amp)
