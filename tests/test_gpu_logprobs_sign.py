"""taps_logprobs: probabilities of at most 1, entropies of at least 0, and exact zeros for the only
value that a mask leaves."""
import numpy as np
import pytest
import torch

import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def score(x, tok, top):
    op = taps.TokenLogProbs(*x.shape, top=top, dtype=taps.BF16 if x.dtype == BF else taps.FP32)
    return op(x, tok)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("mask", [-float("inf"), float("nan"), torch.finfo(BF).min, -1e9, -20000.0])
@pytest.mark.parametrize("V,rows", [(1, 64), (40, 128), (3001, 128), (151936, 9), (30011, 257)])
def test_one_value_left(dtype, mask, V, rows):
    """Its weight is 1 and every other one's 0 (exp of -19,900 at most): logarithm and entropy are 0
    without a rounding, wherever the value stands; V whole, in parts and past the batches."""
    rng = np.random.default_rng(V)
    at = rng.integers(0, V, rows)
    at[:4] = [0, V - 1, V // 2, V // 3]
    values = rng.uniform(-100, 100, rows)
    values[:8] = [0.0, 9.0, -9.0, 1e-30, 99.5, 8.9375, 9.0625, -0.1]
    x = torch.full((rows, 1, V), mask, dtype=dtype, device="cuda")
    tok = torch.from_numpy(at).int().cuda()[:, None]
    x[torch.arange(rows), 0, tok[:, 0].long()] = torch.from_numpy(values).cuda().to(dtype)
    lp, ent, rank, idx, tlp = score(x, tok, 1)
    assert (lp == 0).all() and (ent == 0).all() and (tlp == 0).all()
    assert (rank == 0).all() and torch.equal(idx[..., 0], tok)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V,rows", [(5, 300), (1000, 300), (30011, 257), (151936, 9)])
@pytest.mark.parametrize("second", [None, 0.0, 1e-3, 3.0, 5.6, 12.0, 15.0, 17.0, 30.0])
def test_nothing_above_one(dtype, V, rows, second):
    """Rows whose largest value is alone far above the rest, or beside a second one just so much
    smaller that its weight is about what fp32 resolves; ordinary rows."""
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(rows, 1, V, generator=g, device="cuda")
    if second is not None:
        x -= 40
        x[:, 0, V // 2] = torch.rand(rows, generator=g, device="cuda") * 40 + 5
        x[:, 0, V // 3] = x[:, 0, V // 2] - second
    x = x.to(dtype)
    tok = x[:, :, :].float().argmax(-1).int()
    lp, ent, _, _, tlp = score(x, tok, min(V, 5))
    assert (lp <= 0).all() and (tlp <= 0).all() and (ent >= 0).all()
    assert torch.equal(tlp[..., 0], lp)
