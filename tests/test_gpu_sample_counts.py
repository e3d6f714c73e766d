"""taps_sample on bf16 rows in which a value occurs as often as 16 bits count, or more often."""
import pytest
import torch

from test_gpu_sample import check, uniform

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
V = 151936
COUNTS = [65535, 65536, 65537, 131072]
# without a bound (the row is read once), and with one that thousands of tokens reach (its
# largest value is known before they are counted)
FILTERS = [(0, 1.0, 0.0), (300, 1.0, 0.0), (70000, 1.0, 0.0), (0, 0.9, 0.0), (0, 0.9, 0.02),
           (100000, 0.6, 0.01), (0, 1.0, 0.001), (50, 1.0, 0.0), (100, 0.7, 0.0)]


def rows(*often, top=12.0):
    """A row of normal values below `top`, with (value, count) pairs at places of their own."""
    g = torch.Generator(device="cuda").manual_seed(len(often))
    x = (torch.randn(V, generator=g, device="cuda") * 2).clamp_(max=top - 1).to(BF)
    at = torch.randperm(V, generator=g, device="cuda")
    x[at[-1]] = top
    n = 0
    for value, count in often:
        x[at[n:n + count]] = value
        n += count
    assert n < V
    return x


@pytest.mark.parametrize("count", COUNTS)
def test_a_value_as_often_as_counters_hold(count):
    """Neighbouring values (counters in both halves of a word), high and low in the row's order,
    and as its largest."""
    step = 2.0 ** -7
    x = torch.stack([rows((v, count), top=max(12.0, v)) for v in
                     (1.0, 1.0 + step, -1.0, -1.0 - step, 12.0, 8.0 + 8 * step, 0.0)])
    for i, (k, p, m) in enumerate(FILTERS):
        check(x[None], uniform(count + i, 1, x.shape[0]), None, [0.9], [k], [p], [m])


def test_several_values_past_the_counters():
    """Both counters of a word, and zeros of both signs that only together are too many."""
    step = 2.0 ** -7
    x = torch.stack([
        rows((1.0, 65536), (1.0 + step, 65536)), rows((1.0 + step, 65536), (1.0 + 2 * step, 65536)),
        rows((1.0, 65535), (1.0 + step, 65536)), rows((1.0, 65536), (1.0 + step, 65535)),
        rows((0.0, 40000), (-0.0, 40000)), rows((0.0, 32768), (-0.0, 32767)),
        rows((0.0, 32768), (-0.0, 32768)), rows((-0.0, 65536)), rows((0.0, 65535), (-0.0, 1)),
        rows((0.0, 70000), (-0.0, 70000), top=0.0),
        torch.zeros(V, dtype=BF, device="cuda"), torch.full((V,), -3.0, dtype=BF, device="cuda"),
    ])
    for i, (k, p, m) in enumerate(FILTERS):
        check(x[None], uniform(i, 1, x.shape[0]), None, [0.9], [k], [p], [m])
