"""taps_sample where very many tokens have weights about one unit (2^-43 of the largest): those
of at most half a unit round to 0 and are never drawn, however many there are."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
V = 1 << 20
# depths below the largest value in octaves, of which 44 is half a unit
NONE, SOME = [44.01, 44.15, 44.3, 44.46, 44.49, 44.6], [43.0, 43.3]
U = np.array([[0.0, 0.5, 1 - 2 ** -24, 1.0]], np.float32)
FILTERS = [dict(), dict(top_p=0.9999), dict(top_p=float(np.float32(1 - 2 ** -24))), dict(top_k=V - 1),
           dict(min_p=1e-30), dict(min_p=1e-30, top_p=0.9999)]


def draw(x, **kw):
    t = {k: torch.tensor([v], dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda")
         for k, v in kw.items()}
    op = taps.TokenSampler(1, U.shape[1], V, dtype=taps.BF16 if x.dtype == BF else taps.FP32)
    tok, pr = op(x.view(1, 1, V).repeat(1, U.shape[1], 1), torch.from_numpy(U).cuda(), **t)
    return tok[0].tolist(), pr[0].double().cpu().numpy()


@pytest.mark.parametrize("octaves", NONE)
@pytest.mark.parametrize("dtype", [BF, FP])
def test_weights_that_round_to_zero_are_never_drawn(dtype, octaves):
    """One token beside a million of weight 0: every number draws it, with probability 1."""
    x = torch.full((V,), -octaves * np.log(2), dtype=torch.float64, device="cuda").to(dtype)
    x[777777] = 0.0
    depth = -float(x[0]) / np.log(2)                       # as rounded to the type
    assert depth > 44
    for kw in FILTERS:
        tok, pr = draw(x, **kw)
        assert tok == [777777] * U.shape[1] and (pr == 1.0).all(), (kw, tok, pr)


@pytest.mark.parametrize("temperature", [0.5, 4.0])
def test_only_weights_above_half_a_unit_are_drawn(temperature):
    """Tokens on both sides of half a unit, hundreds of thousands of each, at the end of the
    rank order: the last token drawn has a weight.  Sums keep the weights to within two units
    each, the largest one is all but 2^-22 of the sum."""
    half = torch.arange(V, device="cuda") % 2 == 0
    for above in SOME:
        x = torch.where(half, -above, -44.2).mul(np.log(2) * temperature).to(FP)
        x[5] = 0.0
        w, _ = oracle.sample_row(x.double().cpu().numpy(), 1.0, temperature=temperature)
        assert w % 2 == 0                                  # the oracle's last one
        for kw in FILTERS[:1] + FILTERS[3:5]:
            tok, pr = draw(x, temperature=temperature, **kw)
            assert tok[0] == 5 and tok[1] == 5 and tok[3] % 2 == 0, (kw, tok)
            # at most 2^20 weights of less than 2^-42 beside the largest
            assert abs(pr[0] - 1.0) <= 2.0 ** -22 + 2.0 ** -24 and pr[3] <= 2.0 ** -42, (kw, pr)
