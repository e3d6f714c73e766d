"""qk_rope_paged's norm where a head's squares leave the range of 32 bits, or eps is tiny or 0."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps
from test_gpu_rope import f64, inputs

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 24), (64, 64), (64, 16)])
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-38, 1e-30, 1e-6, 1e6, 1e30])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_of_any_size(dtype, hd, rot, eps, interleaved):
    """Head h of each row is scaled by a power of two, from values below the smallest normal one
    to 2^118, so that its squares are subnormal, vanish or overflow.  eps is the fp32 number.
    The bound: as for ordinary heads, and what values rounded to subnormal results lose."""
    eps = float(np.float32(eps))
    freq, _ = taps.rope_frequencies(rot, 1e4)
    scales = [-130 if dtype == BF else -146, -126, -100, -76, -70, -66, -64, -63, -60, -50, -30, 0, 30, 50, 60, 63, 64, 80, 118]
    H = len(scales)
    Q, K, V, pos, slots, Kp, Vp, qw, kw = inputs(hd + rot, 9, H, H, hd, 32, dtype, fused=False,
                                                 pad=False)
    s = torch.tensor(scales, dtype=torch.float64, device="cuda")[:, None]
    Q, K = ((t.double() * 2.0 ** s).to(dtype) for t in (Q, K))
    if eps > 0:
        Q[4, 3], K[5, 12] = 0, 0                            # a zero head stays zero
    want = oracle.qk_rope_paged(f64(Q), f64(K), f64(V), pos.cpu().numpy(), slots.cpu().numpy(),
                                f64(freq), 1.0, interleaved, f64(qw), f64(kw), eps, f64(Kp), f64(Vp))
    op = taps.PagedQKRope(H, H, hd, 32, freq, dtype=taps.BF16 if dtype == BF else taps.FP32,
                          interleaved=interleaved, eps=eps)
    got = op(Q, K, V, pos, slots, Kp, Vp, q_norm=qw, k_norm=kw)
    step, least = (2.0 ** -8, 2.0 ** -133) if dtype == BF else (2.0 ** -24, 2.0 ** -149)
    for name, a, ref, mag in (("Q", got, want[0], want[3]), ("K", Kp, want[1], want[4])):
        a = f64(a)
        assert np.isfinite(a).all(), name
        err = np.abs(a - ref)
        assert (err <= np.abs(ref) * step + mag * 2.0 ** -19 + 4 * least).all(), name


def test_zero_heads_and_infinities():
    """eps 0: a zero head has no direction (0 / 0), and infinities leave NaN in their own places."""
    freq, _ = taps.rope_frequencies(16, 1e4)
    Q, K, V, pos, slots, Kp, Vp, qw, kw = inputs(3, 4, 4, 2, 64, 32, FP, fused=False, pad=False)
    Q[0, 1] = 0
    Q[1, 2, 40] = float("inf")
    Q[2, 3, 50] = float("nan")
    out = taps.PagedQKRope(4, 2, 64, 32, freq, dtype=taps.FP32, eps=0.0)(
        Q, K, V, pos, slots, Kp, Vp, q_norm=qw, k_norm=kw)
    bad = torch.isnan(out)
    assert bad[0, 1].all() and bad[2, 3].all()
    assert bad[1, 2, 40] and (out[1, 2].nan_to_num(0) == 0).all() and bad[1, 2].sum() == 1
    bad[0, 1], bad[1, 2], bad[2, 3] = False, False, False
    assert not bad.any()
