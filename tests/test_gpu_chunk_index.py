"""chunk_attn_paged of more than 256 requests: every entry of their index that is read was written."""
import numpy as np
import pytest
import torch

import paper_2606_00487_amd as taps
from test_gpu_chunk import BF, FP, call, case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fill", [0x00, 0x7F, 0xFF])
@pytest.mark.parametrize("B,most,long", [(257, 4, 0), (300, 4, 5000), (1100, 2, 3000)])
def test_scratch_of_any_content(dtype, fill, B, most, long):
    rng = np.random.default_rng(B)
    lens = [(int(a), int(a + c)) for a, c in zip(rng.integers(0, most, B), rng.integers(0, 60, B))]
    lens[0], lens[B - 1] = (0, 0), (0, 7)
    if long:                                              # some caches are cut, some requests not
        lens[B // 2], lens[B // 3] = (3, long), (30, long // 2)
    Q, K, V, table, start, kv, max_len = case(B, lens, 4, 2, 64, 32, dtype)
    op, want = call(Q, K, V, table, start, kv, max_len)
    n = op._ws_bytes(Q.shape[0])
    assert n >= 16 * (B + 1)
    ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
    O = torch.full_like(want, 7.0)
    st = op.lib.chunk_attn_paged(
        Q.data_ptr(), Q.stride(0), K.data_ptr(), V.data_ptr(), K.shape[0], 32, table.data_ptr(),
        table.shape[1], start.data_ptr(), kv.data_ptr(), B, Q.shape[0], 4, 2, 64, max_len, 0,
        taps.BF16 if dtype == BF else taps.FP32, op.scale, O.data_ptr(), ws.data_ptr(), n,
        torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(O, want)
