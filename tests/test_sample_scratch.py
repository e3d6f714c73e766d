"""taps_sample takes no scratch: its size is 0 everywhere, and the call looks at none (host
checks; no kernel runs here)."""
import ctypes

import pytest

from paper_2606_00487_amd import _lib

F = 1 << 20    # aligned, never dereferenced: every case stops before a launch


@pytest.mark.parametrize("batch,budget,vocab,dtype", [
    (1, 1, 1, 0), (16, 128, 151936, 0), (64, 1, 50257, 1), (2048, 512, 1 << 20, 1), (0, 1, 10, 0), (-1, 0, 0, 9)])
def test_scratch_size(lib, batch, budget, vocab, dtype):
    assert lib.taps_sample_workspace_bytes(batch, budget, vocab, dtype) == 0


@pytest.mark.parametrize("ws,ws_bytes", [(None, 0), (F + 3, 1), (None, 1 << 40)])
def test_scratch_is_not_looked_at(lib, ws, ws_bytes):
    st = _lib.Sampling(None, None, None, None)
    call = lambda batch, u: lib.taps_sample(F, 10, batch, 1, 10, 0, None, ctypes.byref(st), u, F,  # noqa: E731
                                            None, ws, ws_bytes, None)
    assert call(0, F) == _lib.TAPS_OK and call(1, F + 2) == _lib.TAPS_ERR_INVALID_ARG
