"""taps_logprobs against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def peaked(seed, *shape, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(*shape, generator=g, device="cuda") * 3
    at = torch.randint(shape[-1], (*shape[:-1], 20), generator=g, device="cuda")
    x.scatter_add_(-1, at, torch.linspace(9, 1, 20, device="cuda").expand(*shape[:-1], 20).contiguous())
    tok = torch.where(torch.rand(shape[:-1], generator=g, device="cuda") < 0.6, at[..., 0],
                      torch.randint(shape[-1], shape[:-1], generator=g, device="cuda"))
    return x.to(dtype), tok.int()


def check(x, tok, top=0, n=None):
    """Ranks and indices equal; |error| of the logarithm of the sum: a rounding per value of a
    thread (vocab / 512 and 40 for the batches), three units for exponent and exponential; of the
    result: half a step.  Entropy: the same of its terms, each within |x - x_0| and the 16 ln 2
    that a thread's reference may be away."""
    B, N, V = x.shape
    op = taps.TokenLogProbs(B, N, V, top=top, dtype=taps.BF16 if x.dtype == BF else taps.FP32)
    got = [t.cpu().numpy() for t in op(x, tok, n)]
    rel = (V / 512 + 43) * 2.0 ** -24
    for b in range(B):
        for i in range(N):
            lp, ent, rank, idx, tlp = (t[b, i] for t in got)
            if n is not None and i >= int(n[b]):
                assert (lp, ent, rank) == (0, 0, -1) and (idx == -1).all() and (tlp == 0).all()
                continue
            w = oracle.logprobs_row(x[b, i].double().cpu().numpy(), int(tok[b, i]), top)
            assert rank == w[2], (b, i, rank, w[2])
            assert np.array_equal(idx, w[3]), (b, i, idx, w[3])
            for a, r in [(lp, w[0])] + list(zip(tlp, w[4])):
                assert a == r or abs(a - r) <= rel + abs(r) * 2.0 ** -24, (b, i, a, r)
            assert abs(ent - w[1]) <= rel * (1 + w[5] + 12) + abs(w[1]) * 2.0 ** -24, (b, i, ent, w[1])
    return got


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V,top", [(1, 1), (2, 2), (7, 5), (8, 8), (64, 20), (1000, 5), (1003, 20),
                                   (4096, 1), (16384, 0), (32001, 64), (151936, 5)])
def test_vocabularies(dtype, V, top):
    x, tok = peaked(V, 2, 3, V, dtype=dtype)
    check(x, tok, top)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_special_values(dtype):
    V = 5000
    x, tok = peaked(1, 16, 1, V, dtype=dtype)
    lowest = torch.finfo(dtype).min
    x[0, 0, :] = -INF                                    # nothing is left
    x[1, 0, :] = NAN
    x[2, 0, 17] = INF
    x[3, 0, [5, 4000]] = INF
    x[4, 0, 100:] = -INF                                 # a mask
    x[5, 0, 3:] = -INF                                   # fewer than `top` are left
    x[6, 0, :] = lowest
    x[7, 0, 10:] = lowest                                # a mask of the type's lowest value
    x[8, 0, ::3] = NAN
    x[9, 0, :] = NAN
    x[9, 0, 4321] = -2.0
    x[10, 0, :] = 1.5                                    # all equal
    x[11, 0, :2500], x[11, 0, 2500:] = 0.0, -0.0
    x[12, 0, :] = torch.finfo(dtype).max
    x[13, 0, 7] = torch.finfo(dtype).max
    x[14, 0, 1:] = -INF
    x[15, 0, 2000:] = NAN
    x[15, 0, :2000] = -INF
    for t in (0, 17, 4321, 4999, 5):
        tok.fill_(t)
        check(x, tok, 20)


def test_signalling_nan():
    x, tok = peaked(2, 2, 1, 3000)
    x.view(torch.int16)[0, 0, 5::9] = 0x7F81             # NaN with the quiet bit clear
    check(x, tok, 5)
    y, tok = peaked(3, 2, 1, 3000, dtype=FP)
    y.view(torch.int32)[0, 0, 5::9] = 0x7F800001
    check(y, tok, 5)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_many_equal_values(dtype):
    """More ties than the candidates' room, at the top and at the bound."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randint(0, 3, (3, 1, 20001), generator=g, device="cuda").to(dtype)
    x[1, 0, :7] = 9.0
    tok = torch.tensor([[20000], [3], [11]], dtype=torch.int32, device="cuda")
    check(x, tok, 30)
    x = torch.arange(20001, device="cuda").repeat(2, 1, 1).to(dtype)     # rising, falling
    x[1] = x[1].flip(-1)
    check(x, tok[:2], 30)


def test_tokens_outside_and_rows_left_out():
    x, tok = peaked(5, 3, 4, 777, dtype=FP)
    tok[0, 0], tok[0, 1], tok[1, 2] = -1, 777, 2 ** 31 - 1
    tok[1, 0] = -(2 ** 31)
    n = torch.tensor([2, 4, 0], dtype=torch.int32, device="cuda")
    check(x, tok, 3, n)
    check(x, tok, 0, n)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_views_of_odd_vocabularies(dtype):
    """Rows that begin anywhere inside 16 bytes; rows of a padded vocabulary."""
    base, _ = peaked(6, 1, 40, 1013, dtype=dtype)
    tok = torch.randint(0, 1013, (1, 40), device="cuda", dtype=torch.int32)
    check(base, tok, 4)
    check(base[:, 3:], tok[:, 3:].contiguous(), 4)
    wide, _ = peaked(7, 5, 3, 1024, dtype=dtype)
    check(wide[..., :1000], tok[:, :15].reshape(5, 3).clamp(max=999), 4)


def test_large_and_small_logits():
    x, tok = peaked(8, 4, 1, 9000, dtype=FP)
    x[0] *= 1e4
    x[1] += 3e4
    x[2] *= 1e-6
    x[3] = torch.linspace(-80, 80, 9000, device="cuda")
    check(x, tok, 8)


def test_same_bits_on_streams_and_in_graphs():
    x, tok = peaked(9, 4, 8, 50001)
    op = taps.TokenLogProbs(4, 8, 50001, top=7)
    want = op(x, tok)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = op(x, tok)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = op(x, tok)
    for i in range(3):
        x.copy_(peaked(10 + i, 4, 8, 50001)[0])
        eager = op(x, tok)
        for o in outs:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


def test_no_requests():
    out = taps.TokenLogProbs(0, 3, 100, top=2)(torch.empty(0, 3, 100, dtype=BF, device="cuda"),
                                              torch.empty(0, 3, dtype=torch.int32, device="cuda"))
    assert [tuple(t.shape) for t in out] == [(0, 3)] * 3 + [(0, 3, 2)] * 2


@pytest.mark.parametrize("dtype", [BF, FP])
def test_special_values_of_rows_in_parts(dtype):
    """Few rows of a large vocabulary are cut into parts: parts without values, with infinities, with
    fewer than `top` values, the token in each of them."""
    V = 70001
    x, tok = peaked(31, 13, 1, V, dtype=dtype)
    x[0, 0, :] = -INF
    x[1, 0, :] = NAN
    x[2, 0, 40000] = INF
    x[3, 0, [5, 69999]] = INF
    x[4, 0, 100:] = -INF
    x[5, 0, :-7] = -INF
    x[6, 0, :35000] = NAN
    x[7, 0, 30000:] = torch.finfo(dtype).min
    x[8, 0, :] = NAN
    x[8, 0, 50000] = -2.0
    x[9, 0, :] = -3.25                                   # all equal: the first ones
    x[10, 0, :35000], x[10, 0, 35000:] = -0.0, 0.0
    x[11, 0, 35000:] = -INF
    x[11, 0, :35000] = NAN
    for t in (0, 20000, 40000, 70000, -1):
        tok.fill_(t)
        check(x, tok, 20)
    n = torch.tensor([i % 2 for i in range(13)], dtype=torch.int32, device="cuda")
    check(x, tok, 3, n)


@pytest.mark.parametrize("rows", [1, 2, 3, 31, 64, 65, 128, 129, 257])
def test_numbers_of_rows_around_the_cut(rows):
    x, tok = peaked(rows, rows, 1, 50021)
    check(x, tok, 2)


def test_rows_past_32_bits():
    """Rows whose bytes lie past 4 GB."""
    x, tok = peaked(41, 9, 1, 1000)
    far = torch.empty(9, 1 << 28, dtype=BF, device="cuda")
    far[:, :1000] = x[:, 0]
    got = check(far[:, None, :1000], tok, top=8)
    want = check(x, tok, top=8)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


def test_scratch_that_holds_nan():
    x, tok = peaked(42, 3, 1, 70001)
    op = taps.TokenLogProbs(3, 1, 70001, top=9)
    want = op(x, tok)
    ws = torch.full((op.ws_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
    got = [torch.full_like(t, 7) for t in want]
    st = op.lib.taps_logprobs(x.data_ptr(), 70001, 3, 1, 70001, taps.BF16, None, tok.data_ptr(), 9,
                              *(t.data_ptr() for t in got), ws.data_ptr(), op.ws_bytes,
                              torch.cuda.current_stream().cuda_stream)
    assert st == 0 and op.ws_bytes > 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("mask", [-INF, torch.finfo(BF).min, -1e9, -20000.0])
@pytest.mark.parametrize("V,rows", [(151936, 2), (30011, 3)])
def test_masks_that_leave_few_values(dtype, mask, V, rows):
    """0 to 100 values left, alternatives among them and in the mask; V in parts and whole."""
    left = [0, 1, 5, 40, 63, 64, 65, 100][:rows * 4]
    for top in (1, 5, 20, 33, 64):
        x, tok = peaked(43, len(left), 1, V, dtype=dtype)
        rng = np.random.default_rng(top)
        for b, n in enumerate(left):
            keep = torch.from_numpy(rng.choice(V, n, replace=False)).cuda()
            row = torch.full((V,), mask, dtype=dtype, device="cuda")
            row[keep] = x[b, 0, keep]
            x[b, 0] = row
            if n:
                tok[b, 0] = int(keep[0])
        check(x, tok, top=top)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("top", [20, 32, 33, 64])
@pytest.mark.parametrize("distinct,equal", [(0, 600), (10, 600), (10, 5000), (31, 513), (500, 600),
                                            (2000, 3000), (64, 20000), (5, 511)])
def test_more_values_at_the_bound_than_candidates(dtype, top, distinct, equal):
    """A few values above many equal ones, anywhere in the row; the rest far below."""
    V = 40000
    rng = np.random.default_rng(distinct + equal + top)
    x = torch.from_numpy(rng.normal(size=(3, 1, V)) - 40).cuda().to(dtype)
    for b in range(3):
        at = torch.from_numpy(rng.permutation(V)[:distinct + equal]).cuda()
        if b == 2:
            at = at.sort().values          # the distinct ones first
        x[b, 0, at[:distinct]] = (3 + torch.arange(distinct, device="cuda") / 64).to(dtype)
        x[b, 0, at[distinct:]] = 2.0
    tok = torch.tensor([[5], [at[0].item()], [at[-1].item()]], dtype=torch.int32, device="cuda")
    check(x, tok, top=top)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V", [1, 63, 64, 65, 200, 511, 512, 513, 700, 2000])
def test_all_alternatives_of_small_vocabularies(dtype, V):
    x, tok = peaked(44, 4, 1, V, dtype=dtype) if V >= 20 else (
        torch.ones(4, 1, V, dtype=dtype, device="cuda"),
        torch.zeros(4, 1, dtype=torch.int32, device="cuda"))
    x[1] = -INF
    x[2, 0, : V // 2] = NAN
    x[3, 0, V // 2:] = INF
    check(x, tok, top=min(V, 64))


def test_sixty_four_alternatives_of_many_rows():
    x, tok = peaked(45, 300, 1, 20000)
    check(x, tok, top=64)
    check(x.float(), tok, top=64)
