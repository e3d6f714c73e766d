"""Where taps_sample's logits may begin (host checks; no kernel runs here)."""
import ctypes

import pytest

from paper_2606_00487_amd import _lib

F = 1 << 20    # aligned, never dereferenced: every case stops before a launch


@pytest.mark.parametrize("dtype,vocab,offset", [
    (_lib.TAPS_BF16, 1001, 1), (_lib.TAPS_BF16, 1001, 15), (_lib.TAPS_BF16, 1000, 2),
    (_lib.TAPS_BF16, 1000, 8), (_lib.TAPS_FP32, 1001, 2), (_lib.TAPS_FP32, 1001, 1),
    (_lib.TAPS_FP32, 1000, 4), (_lib.TAPS_FP32, 1000, 8),
])
def test_refuses_bases_between_elements_or_units(lib, dtype, vocab, offset):
    st = _lib.Sampling(None, None, None, None)
    assert lib.taps_sample(F + offset, vocab, 1, 1, vocab, dtype, None, ctypes.byref(st), F, F, None,
                           None, 0, None) == _lib.TAPS_ERR_INVALID_ARG
