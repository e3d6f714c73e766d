"""decode_attn_paged with one workgroup per request, KV head and group of query heads (short
caches; no scratch), against attention in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_decode import BF, FP, case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("batch,max_len,Hq,Hkv,hd,page_rows", [
    # at most 256 rows, any batch
    (1, 256, 8, 2, 128, 32), (9, 256, 34, 2, 128, 64), (5, 200, 48, 1, 64, 128), (3, 1, 4, 4, 128, 32),
    # batches that fill the chip, at most 1024 rows: up to eight units of 128 keys
    (64, 1024, 16, 8, 64, 64), (64, 1024, 16, 8, 128, 32), (300, 900, 34, 1, 128, 64),
    (300, 1000, 34, 1, 64, 32), (130, 1024, 8, 4, 128, 4096), (520, 700, 1, 1, 64, 32),
])
def test_requests_as_they_are(dtype, batch, max_len, Hq, Hkv, hd, page_rows):
    """Ragged batches with empty requests, the longest at max_len, unit and tile borders."""
    rng = np.random.default_rng([batch, max_len, hd])
    lens = [int(n) for n in rng.integers(0, max_len + 1, batch)]
    edge = [max_len, 0, max_len - 1, 1, 128, 127, 129, 32, 33, 256, 512, 640, 1023]
    for b, n in enumerate(edge[:batch]):
        lens[b] = min(n, max_len)
    if batch > 20:
        lens[-1] = 0
    op, _ = check(*case(batch + hd, lens, Hq, Hkv, hd, page_rows, dtype, max_len=max_len))
    assert op.ws_bytes == 0                                # the plan that this file is about
