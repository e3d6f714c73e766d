"""chunk_attn_paged in fp32: scores far from 0 in caches that are cut."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,kv,G", [(1, 1024, 4), (16, 1024, 4), (3, 700, 1), (1, 1500, 16)])
@pytest.mark.parametrize("level", [0, 1000, -1000])
def test_scores_of_any_level(hd, n, kv, G, level):
    """Scores near 32 * level, of which the first dim alone gives an exact product (a power of two
    times at most 18 bits), that rise by 2 from the first part's keys to the last ones': the softmax
    does not depend on the level, so neither may its error.  V changes sign between the parts.
    |error| over A = sum of the weights times |v|: the exponent (s - m) scale log2 e is at most 6 + 8
    in size (the scores' spread, and how far a reference may lag), off by two roundings and the
    scale's own, 3 * 14 * 2^-24, an exponential good to two units: together below 2^-18, in the
    weights and in their sum; the sums, a rounding for each of a part's at most 192 keys and its
    join's 16, twice: 2^-15."""
    rng = np.random.default_rng(kv + G)
    pr, Hkv, scale = 64, 2, 0.125
    pages = -(-kv // pr)
    rows = np.arange(pages * pr)
    K = torch.from_numpy(rng.normal(size=(pages * pr, Hkv, hd))).float()
    u = rng.integers(0, 16, (pages * pr, Hkv)) + (16 * rows // kv)[:, None]
    K[..., 0] = torch.from_numpy(level + u / 256.0).float()
    V = torch.from_numpy(rng.normal(size=K.shape) + (1 - 2 * (rows // 128 % 2))[:, None, None] * 3).float()
    Q = torch.zeros(n, Hkv * G, hd)
    Q[..., 0] = 256.0
    K, V = K.unflatten(0, (pages, pr)), V.unflatten(0, (pages, pr))
    table, start = np.arange(pages, dtype=np.int32)[None], np.array([0, n], dtype=np.int32)
    op = taps.PagedChunkAttention(1, n, Hkv * G, Hkv, hd, kv, pr, dtype=taps.FP32, scale=scale)
    O = op(Q.cuda(), K.cuda(), V.cuda(), torch.from_numpy(table).cuda(),
           torch.from_numpy(start).cuda(), torch.tensor([kv], dtype=torch.int32, device="cuda"))
    assert op._ws_bytes(n) > 0                              # (cut)
    ref, A, _, _ = oracle.chunk_attention_paged(Q.double().numpy(), K.double().numpy(),
                                                V.double().numpy(), table, start, [kv], scale)
    err = np.abs(O.double().cpu().numpy() - ref)
    lim = np.abs(ref) * 2.0 ** -24 + A * (2.0 ** -17 + 2.0 ** -15)
    print(f"max error {err.max():.3e}, at most {np.max(err / lim):.3f} of its bound", flush=True)
    assert (err <= lim).all()
