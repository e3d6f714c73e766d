"""taps_sample against the sorted row with integer weights: tokens equal, probabilities to
their rounding."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def dev(a, dt=torch.float32):
    return None if a is None else torch.tensor(np.asarray(a), dtype=dt, device="cuda")


def check(x, u, n=None, T=None, k=None, p=None, m=None, logits=None):
    """x: [B, N, V] on the GPU; the settings are lists of B values."""
    B, N, V = x.shape
    op = taps.TokenSampler(B, N, V, dtype=taps.BF16 if x.dtype == BF else taps.FP32)
    i32 = torch.int32
    T, p, m, u = (None if a is None else np.asarray(a, np.float32) for a in (T, p, m, u))
    tok, pr = op(x if logits is None else logits, dev(u), dev(n, i32), temperature=dev(T),
                 top_k=dev(k, i32), top_p=dev(p), min_p=dev(m))
    wt, wp = oracle.sample(x.double().cpu().numpy(), u, n, T, k, p, m)
    np.testing.assert_array_equal(tok.cpu().numpy(), wt)
    # a weight is off by one unit (2^-43) at most, its rounding to float by 2^-24 of it
    err = np.abs(pr.double().cpu().numpy() - wp)
    assert (err <= 2.0 ** -24 * wp + 2.0 ** -40).all(), err.max()
    return tok, pr


def normal(seed, B, N, V, dtype, sigma=3.0, raised=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, N, V, generator=g, device="cuda") * sigma
    if raised:
        at = torch.randint(V, (B, N, raised), generator=g, device="cuda")
        x.scatter_add_(2, at, torch.linspace(9, 1, raised, device="cuda").expand(B, N, raised).contiguous())
    return x.to(dtype)


def uniform(seed, B, N):
    return np.random.default_rng(seed).random((B, N)).astype(np.float32) * np.float32(1 - 2 ** -24)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 1000, 4099, 50257])
def test_settings_by_request(dtype, V):
    """Every filter and their mixes, one request each, over odd and tiny vocabularies."""
    T = [1.0, 0.7, 1.3, 0.6, 1.0, 0.9, 0.0, -1.0, NAN, 1.0, 2.0, 0.05, 50.0, 1.0]
    k = [0, 1, 20, 50, 0, 3, 5, 0, 0, -4, 2 ** 31 - 1, 0, 700, V]
    p = [1.0, 1.0, 1.0, 0.8, 0.9, 0.5, 0.5, 0.9, 0.2, NAN, 0.999, 0.95, 0.97, 0.0]
    m = [0.0, 0.0, 0.0, 0.0, 0.0, 0.3, 0.1, 0.0, 0.0, 0.05, 0.0, 0.0, 0.5, NAN]
    B, N = len(T), 3
    check(normal(V, B, N, V, dtype, raised=min(V, 30)), uniform(V, B, N), None, T, k, p, m)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sigma", [0.0, 0.01, 0.5, 8.0, 300.0])
def test_flat_and_steep_rows(dtype, sigma):
    """From all-equal rows (nothing but ties) to rows with one token; large kept sets."""
    T, k = [1.0] * 6, [0, 0, 0, 3000, 17, 0]
    p, m = [1.0, 0.9, 0.3, 1.0, 0.7, 1.0], [0.0, 0.0, 0.0, 0.0, 0.0, 0.6]
    check(normal(3, 6, 4, 20011, dtype, sigma), uniform(4, 6, 4), None, T, k, p, m)


def test_largest_vocabularies():
    check(normal(5, 5, 2, 151936, BF, raised=40), uniform(5, 5, 2), None, [0.7, 1, 1, 0, 1.5],
          [20, 0, 0, 0, 0], [0.8, 0.95, 1, 1, 0.9], [0, 0, 0, 0, 0.02])
    check(normal(6, 2, 1, 1 << 20, FP), uniform(6, 2, 1), None, [1, 1], [0, 40], [0.9, 1], None)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_random_numbers_at_their_ends(dtype):
    """u of 0, just below 1, 1, beyond and NaN; ties whose borders are exact: 2^-k of them."""
    u = np.array([[0.0, 1 - 2 ** -24, 1.0, 7.0, -2.0, NAN, 0.25, 0.5, 0.75, 0.5 - 2 ** -25]],
                 np.float32)
    x = torch.zeros(1, 10, 64, dtype=dtype, device="cuda")
    tok, pr = check(x, u)
    assert tok[0].tolist() == [0, 63, 63, 63, 0, 0, 16, 32, 48, 31]
    check(x, u, None, None, [16], [0.5], None)
    check(x, u, None, None, None, [0.5], None)
    check(normal(8, 1, 10, 3001, dtype), u)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("filters", [(None, None, None), ([30], None, None), (None, [0.9], None),
                                     (None, None, [0.1]), ([30], [0.5], [0.1])])
def test_rows_with_infinities_nan_and_masks(dtype, filters):
    low = torch.finfo(dtype).min
    V = 300
    x = normal(9, 1, 12, V, dtype)
    x[0, 0] = NAN
    x[0, 1] = -INF
    x[0, 2, 5:] = -INF
    x[0, 3, :-1] = NAN
    x[0, 4, [7, 200]] = INF
    x[0, 5] = low
    x[0, 6, 1:] = low
    x[0, 7, ::2] = NAN
    x[0, 8, :150] = low
    x[0, 9, 0], x[0, 9, 1:] = torch.finfo(dtype).max, low
    x[0, 10], x[0, 10, 3], x[0, 10, 9] = NAN, -INF, -INF
    x[0, 11, ::3], x[0, 11, 1::3] = 0.0, -0.0
    k, p, m = filters
    for s in range(3):
        check(x, uniform(s, 1, 12), None, [0.8], k, p, m)
    check(x, uniform(3, 1, 12), None, [0.0], k, p, m)
    check(x, uniform(4, 1, 12), None, [1e-40], k, p, m)
    check(x, uniform(5, 1, 12), None, [INF], k, p, m)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_past_the_tree_and_padded_vocabularies(dtype):
    """Rows i >= n_nodes are not read and give -1; the logits are a slice of a padded head."""
    B, N, V = 4, 9, 1003
    wide = torch.full((B, N, V + 21), INF, dtype=dtype, device="cuda")
    x = normal(10, B, N, V, dtype)
    wide[..., :V] = x
    n = [9, 0, 4, 1]
    for b in range(B):
        x[b, n[b]:], wide[b, n[b]:] = NAN, NAN
    T, k, p = [1.0, 1.0, 0.6, 0.0], [0, 0, 12, 0], [0.9, 1.0, 0.8, 1.0]
    a = check(x, uniform(11, B, N), n, T, k, p)
    b = check(x, uniform(11, B, N), n, T, k, p, logits=wide[..., :V])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one = wide[:, :1, :V]                                   # a row per request, far apart
    check(x[:, :1], uniform(12, B, 1), None, T, k, p, logits=one)
    check(x[:1], uniform(13, 1, N), n[:1], T[:1], k[:1], p[:1], logits=wide[:1, :, :V])


@pytest.mark.parametrize("k", [1, 2, 15, 16, 17, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049, 5000])
def test_top_k_sizes(k):
    for dtype in (BF, FP):
        x = normal(k, 2, 2, 9001, dtype, 1.0)
        check(x, uniform(k, 2, 2), None, [1.0, 0.4], [k, k], [1.0, 0.9], None)


def test_ties_at_every_border():
    """A handful of distinct values, each thousands of times: every border is among ties."""
    g = torch.Generator(device="cuda").manual_seed(14)
    x = torch.randint(-3, 3, (4, 6, 30000), generator=g, device="cuda").to(BF)
    check(x, uniform(14, 4, 6), None, [1.0, 0.5, 2.0, 1.0], [0, 7000, 0, 100], [0.7, 1.0, 0.99, 0.5],
          [0.0, 0.0, 0.3, 0.0])


def test_graph_replays_and_streams():
    x = normal(15, 2, 8, 50000, BF, raised=30)
    u = dev(uniform(15, 2, 8))
    op = taps.TokenSampler(2, 8, 50000)
    kw = dict(temperature=dev([0.8, 1.0]), top_p=dev([0.9, 0.95]))
    want = op(x, u, **kw)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    graphs, outs = [], []
    for s in (s1, s2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(op(x, u, **kw))
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(4):
        for t, _p in outs:
            t.fill_(-9)
        torch.cuda.synchronize()
        for s, g in ((s1, graphs[0]), (s2, graphs[1])):
            with torch.cuda.stream(s):
                g.replay()
        e = op(x, u, **kw)
        torch.cuda.synchronize()
        for o in (*outs, e):
            assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1])


def test_refuses_wrong_tensors():
    op = taps.TokenSampler(2, 3, 100)
    x, u = torch.zeros(2, 3, 100, dtype=BF, device="cuda"), torch.zeros(2, 3, device="cuda")
    for bad in (x[:, :2], x[..., :99], torch.zeros(2, 5, 100, dtype=BF, device="cuda")[:, :3],
                torch.zeros(2, 3, 200, dtype=BF, device="cuda")[..., ::2]):
        with pytest.raises(ValueError):
            op(bad, u)
    with pytest.raises(TypeError):
        op(x.float(), u)
    with pytest.raises(TypeError):
        op(x, u.double())
    with pytest.raises(TypeError):
        op(x, u, top_k=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError):
        op(x, u, temperature=torch.zeros(3, device="cuda"))
    with pytest.raises(taps.TapsError):
        taps.TokenSampler(1, 1, (1 << 20) + 1)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rows", [3, 40, 65])
def test_long_rows_shared_out(dtype, rows):
    """Few rows of long vocabularies: steep and flat temperatures, values far from 0, whole
    stretches masked, NaN and infinities, the largest value at either end."""
    V = 33000
    x = normal(20 + rows, 1, rows, V, dtype, raised=30)
    x[0, 0, 100:30000] = -INF
    x[0, 1, :32990] = torch.finfo(dtype).min
    x[0, 2, ::5] = NAN
    if rows > 3:
        x[0, 3, 20000], x[0, 3, 7] = INF, INF
        x[0, 4] = NAN
        x[0, 5] += 3000.0
        x[0, 6] -= 3000.0
        x[0, 7] = 0.5
        x[0, 8, -1] = 30.0
        x[0, 9, 0] = 30.0
        x[0, 10] *= 1000.0
        x[0, 11] = -INF
        x[0, 12, 5:] = -INF
    u = uniform(rows, 1, rows)
    for T, k, p, m in ((1.0, 0, 0.9, 0.0), (0.6, 0, 1.0, 0.0), (2.5, 0, 0.97, 0.0), (0.9, 0, 0.9, 0.02),
                       (1e-3, 0, 0.9, 0.0), (0.02, 0, 0.5, 0.0), (300.0, 0, 0.5, 0.0), (1.0, 1000, 0.9, 0.0),
                       (0.8, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.3), (0.0, 0, 1.0, 0.0), (INF, 0, 0.7, 0.0)):
        check(x, u, None, [T], [k], [p], [m])


def test_min_p_borders_with_top_p():
    """min_p and top_p together, on values an equal step apart, so that borders fall on values."""
    for dtype in (BF, FP):
        for V in (500, 40000):
            x = (torch.arange(V, device="cuda") % 97).mul(-0.0625).to(dtype).view(1, 1, V).repeat(1, 8, 1)
            for m in (0.5, 0.0625 / 2, 0.9, 1.0, 1e-3):
                check(x, uniform(V, 1, 8), None, [1.0], None, [0.95], [m])
                check(x, uniform(V + 1, 1, 8), None, [0.25], [90], [0.99], [m])


@pytest.mark.parametrize("sigma", [1e-5, 0.02, 1.0])
@pytest.mark.parametrize("rounded", [False, True])
def test_dense_rows(sigma, rounded):
    """fp32 rows with thousands of values within a few percent of one another's weight, exact
    ties among them where the logits were bf16 once."""
    B, V = 8, 70001
    x = normal(30, B, 3, V, FP, sigma)
    if rounded:
        x = x.to(BF).to(FP)
    T, k = [1.0, 1.0, 10.0, 0.7, 1.0, 1.0, 2.0, 1.0], [0, 0, 0, 500, 30000, V - 1, 1200, 193]
    p, m = [1.0, 0.9, 0.5, 1.0, 0.9, 1.0, 0.3, 1.0], [0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.9, 0.5]
    check(x, uniform(31, B, 3), None, T, k, p, m)
    check(x, uniform(32, B, 3), None, T, k, p, None)
    check(x.repeat(1, 14, 1)[:, :40].contiguous(), uniform(33, B, 40), None, T, k, p, m)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_signalling_nan(dtype):
    """NaN of every kind (quiet, signalling, either sign) in the largest values' places."""
    V = 5000
    x = normal(40, 1, 8, V, dtype)
    bits = [0x7F81, -0x7F, 0x7FC0, -0x40] if dtype == BF else [0x7F800001, -0x7FFFFF, 0x7FC00000, -0x400000]
    for i, b in enumerate(bits):
        x.view(torch.int16 if dtype == BF else torch.int32)[0, :, i::9] = b
        for T, k, p, m in ((1.0, 0, 1.0, 0.0), (0.7, 40, 0.9, 0.0), (1.0, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0),
                           (1.0, 0, 1.0, 0.1), (1.0, 700, 0.9, 0.01)):
            check(x, uniform(41 + i, 1, 8), None, [T], [k], [p], [m])


@pytest.mark.parametrize("T", [1e-38, 1e-6, 1e4, 3e38])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_extreme_temperatures(dtype, T):
    """Temperatures whose weights are one-hot, or so flat that a bin holds the whole row."""
    x = normal(42, 1, 6, 4000, dtype)
    x[0, 1] *= 1e30
    x[0, 2] *= 1e-30
    x[0, 3, :2000] = -INF
    for k, p, m in ((0, 1.0, 0.0), (0, 0.6, 0.0), (300, 1.0, 0.0), (300, 0.5, 0.0), (0, 1.0, 0.999), (5, 0.9, 0.5)):
        check(x, uniform(43, 1, 6), None, [T], [k], [p], [m])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rows", [8, 264])
def test_late_largest_values(dtype, rows):
    """Rows whose first values say little about the largest: masked, tiny, negative, NaN, or
    thousands of times smaller than a later one."""
    V = 20000
    x = normal(50, 1, 8, V, dtype)
    x[0, 0, :15000] = -INF
    x[0, 1, :15000] = torch.finfo(dtype).min
    x[0, 2, :15000] *= 1e-6
    x[0, 3, :] = -x[0, 3].abs() * 100
    x[0, 3, 17000:17010] = -0.0
    x[0, 4, 19990] = 60000.0
    x[0, 4, 19991:] = 59904.0
    x[0, 5, :15000] = NAN
    x[0, 6, :] *= 1e-3
    x[0, 6, 12345], x[0, 6, 18001] = 500.0, 500.0
    x[0, 7, :15000], x[0, 7, 15000:] = -1e30, x[0, 7, 15000:] - 1e4
    B = rows // 8
    xs, u = x.repeat(B, 1, 1), uniform(51, B, 8)
    u[1:] = u[0]                               # (one oracle row stands for its repeats)
    for T, k, p, m in ((1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.3, 900, 0.95, 0.0), (2.0, 0, 0.9, 0.02)):
        want, wp = check(x, u[:1], None, [T], [k], [p], [m])
        if B > 1:
            op = taps.TokenSampler(B, 8, V, dtype=taps.BF16 if dtype == BF else taps.FP32)
            full = lambda v, t=torch.float32: torch.full((B,), v, dtype=t, device="cuda")  # noqa: E731
            tok, pr = op(xs, dev(u), None, temperature=full(T), top_k=full(k, torch.int32),
                         top_p=full(p), min_p=full(m))
            assert torch.equal(tok, want.expand(B, 8)) and torch.equal(pr, wp.expand(B, 8))
