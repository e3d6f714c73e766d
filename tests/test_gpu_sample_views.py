"""taps_sample on views of logits whose first row begins anywhere: requests and positions left
out of an odd vocabulary's logits need no copy."""
import pytest
import torch

import paper_2606_00487_amd as taps

from test_gpu_sample import BF, FP, check, normal, uniform

pytestmark = pytest.mark.gpu

SETTINGS = [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (0.9, 20, 0.9, 0.0), (1.0, 700, 1.0, 0.0),
            (1.0, 0, 1.0, 0.05), (0.0, 0, 1.0, 0.0)]


def sampled(view, seed):
    B, N, _ = view.shape
    for i, (T, k, p, m) in enumerate(SETTINGS):
        check(view.contiguous().clone(), uniform(seed + i, B, N), None, [T] * B, [k] * B, [p] * B, [m] * B,
              logits=view)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V", [1, 3, 9, 63, 1001, 50257])
def test_requests_left_out(dtype, V):
    x = normal(V, 6, 2, V, dtype)
    for first in (1, 2, 3, 5):
        sampled(x[first:], 10 * first)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V", [5, 63, 1001, 50257])
@pytest.mark.parametrize("length", [2, 4, 8, 9])
def test_last_positions(dtype, V, length):
    """The last position's logits of a whole sequence: [:, -1:]."""
    sampled(normal(V + length, 3, length, V, dtype)[:, -1:], length)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_views_inside_padded_rows(dtype):
    """An odd part of each row, from an odd place on."""
    wide = normal(4, 3, 5, 2048, dtype)
    for start, V in ((1, 999), (3, 1001), (7, 2041 if dtype == BF else 2039)):
        sampled(wide[..., start:start + V], start)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_aligned_vocabularies_keep_aligned_rows(dtype):
    """Rows of whole 16-byte units have to begin at one."""
    flat = torch.zeros(2 * 1024 + 8, dtype=dtype, device="cuda")
    op = taps.TokenSampler(2, 1, 1024, dtype=taps.BF16 if dtype == BF else taps.FP32)
    u = torch.zeros(2, 1, device="cuda")
    for off in (1, 2, 3):
        with pytest.raises(taps.TapsError):
            op(flat[off:off + 2048].view(2, 1, 1024), u)
