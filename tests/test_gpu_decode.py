"""decode_attn_paged against attention in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def case(seed, lens, Hq, Hkv, hd, page_rows, dtype, max_len=None, extra=3, scale_q=1.0):
    """Pages in random order; everything that belongs to no request is NaN."""
    rng = np.random.default_rng(seed)
    B, max_len = len(lens), max_len or max(max(lens), 1)
    need = [-(-n // page_rows) for n in lens]
    pages, width = sum(need) + extra, -(-max_len // page_rows) + 1
    ids = rng.permutation(pages)
    table = rng.choice([-5, 2 ** 31 - 1, pages], (B, width))      # never followed
    own = torch.zeros(pages, page_rows, dtype=torch.bool)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = ids[at:at + m]
        for j in range(m):
            own[ids[at + j], :lens[b] - j * page_rows] = True
        at += m
    g = torch.Generator(device="cuda").manual_seed(seed)
    Q = (torch.randn(B, Hq, hd, generator=g, device="cuda") * scale_q).to(dtype)
    K = torch.randn(pages, page_rows, Hkv, hd, generator=g, device="cuda").to(dtype)
    V = torch.randn(pages, page_rows, Hkv, hd, generator=g, device="cuda").to(dtype)
    K[~own], V[~own] = float("nan"), float("nan")
    return (Q, K, V, torch.tensor(table, dtype=torch.int32, device="cuda"),
            torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len)


def reference(Q, K, V, table, lens, scale):
    h = lambda x: x.double().cpu().numpy()  # noqa: E731
    with np.errstate(invalid="ignore"):
        return oracle.decode_attention_paged(h(Q), h(K), h(V), table.cpu().numpy(),
                                             lens.cpu().numpy(), scale)


def bound(ref, A, D, lens, hd, scale, dtype):
    """|error| of the outputs: the last rounding (half a step), and times A = sum of the weights
    times |v|: the scores' error (hd products and sums of q k, the exponent's own roundings, an
    exponential good to two units), twice since it enters the weights and their sum; one rounding
    per key in the sums of weights and of outputs; bf16: the 2^-17 that two bf16 values leave of
    a weight."""
    n = lens[:, None, None].astype(np.float64)
    score = scale * D[..., None] * (hd + 4) * 2.0 ** -24 + 64 * 2.0 ** -24
    rel = 2 * score + 2 * (n + 64) * 2.0 ** -24 + (2.0 ** -16 if dtype == BF else 0.0)
    return np.abs(ref) * (2.0 ** -8 if dtype == BF else 2.0 ** -24) + A * rel + 1e-30


def check(Q, K, V, table, lens, max_len, scale=None, out=None):
    B, Hq, hd = Q.shape
    op = taps.PagedDecodeAttention(B, Hq, K.shape[2], hd, max_len, K.shape[1],
                                   dtype=taps.BF16 if Q.dtype == BF else taps.FP32, scale=scale)
    O = op(Q, K, V, table, lens, out=out)
    n = lens.clamp(0, max_len)
    ref, A, D = reference(Q, K, V, table, n, op.scale)
    got = O.double().cpu().numpy()
    assert np.isfinite(got).all()
    err = np.abs(got - ref)
    lim = bound(ref, A, D, n.cpu().numpy(), hd, op.scale, Q.dtype)
    print(f"max error {err.max():.3e}, at most {np.max(err / lim):.3f} of its bound", flush=True)
    assert (err <= lim).all()
    return op, O


LENS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (10, 2), (16, 1), (34, 2), (48, 1)])
def test_lengths_and_head_layouts(dtype, hd, Hq, Hkv):
    check(*case(Hq + hd, LENS, Hq, Hkv, hd, 32, dtype))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("page_rows", [32, 64, 256, 4096])
def test_pages(dtype, page_rows):
    check(*case(page_rows, [5000, 0, 4097, 1, 2049], 8, 2, 128, page_rows, dtype))


@pytest.mark.parametrize("lens,max_len,Hq,Hkv,hd,dtype", [
    ([8192], 8192, 32, 8, 128, BF), ([8191], 8192, 4, 1, 64, BF), ([2047], 4000, 32, 8, 128, FP),
    ([30000, 17], 32768, 8, 1, 128, BF), ([1], 20000, 8, 2, 128, BF), ([0, 0], 20000, 8, 2, 64, FP),
    ([9000] + [40] * 70, 9000, 8, 8, 64, BF),
])
def test_splits(lens, max_len, Hq, Hkv, hd, dtype):
    """Long caches, which are cut and joined; grids sized for far more than the requests hold."""
    check(*case(len(lens) + max_len, lens, Hq, Hkv, hd, 64, dtype, max_len=max_len))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_large_scores(dtype):
    """Queries 40 times as large: one key takes nearly all the weight, the reference moves."""
    check(*case(5, [1000, 33, 700], 8, 2, 128, 32, dtype, scale_q=40.0))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_lowest_values_and_scale(dtype):
    """Scores at the far end of the range (values of -3e38 in one key dim) have no weight."""
    Q, K, V, table, lens, m = case(6, [300, 70], 8, 2, 64, 32, dtype)
    K[..., 0] = 0.0
    Q[..., 0] = 1.0
    b0 = table[0, :2].long()
    K[b0, :, :, 0] = -3e38
    check(Q, K, V, table, lens, m, scale=0.3)


def test_lengths_are_clamped():
    Q, K, V, table, lens, m = case(7, [200, 64, 90], 8, 2, 128, 32, BF)
    op = taps.PagedDecodeAttention(3, 8, 2, 128, 200, 32)
    want = op(Q, K, V, table, torch.tensor([200, 0, 90], dtype=torch.int32, device="cuda"))
    got = op(Q, K, V, table, torch.tensor([10 ** 9, -3, 90], dtype=torch.int32, device="cuda"))
    assert torch.equal(want, got) and (got[1] == 0).all()


def test_strided_queries_and_out():
    Q, K, V, table, lens, m = case(8, [100, 333, 64], 8, 2, 128, 32, BF)
    wide = torch.full((3, 14, 128), float("nan"), dtype=BF, device="cuda")
    wide[:, 2:10] = Q
    out = torch.empty_like(Q)
    _, a = check(Q, K, V, table, lens, m)
    _, b = check(wide[:, 2:10], K, V, table, lens, m, out=out)
    assert torch.equal(a, b) and b.data_ptr() == out.data_ptr()


def test_values_that_are_not_finite_stay_in_their_request():
    Q, K, V, table, lens, m = case(9, [600, 600, 40], 8, 2, 128, 32, BF)
    V[table[0, 3].long(), 5, 1, 7] = float("nan")
    K[table[2, 0].long(), 3, 0] = float("nan")
    op = taps.PagedDecodeAttention(3, 8, 2, 128, m, 32)
    O = op(Q, K, V, table, lens).float()
    bad = torch.isnan(O)
    assert bad[0, 4:, 7].all() and int(bad[0].sum()) == 4       # that dim of that head's queries
    assert not bad[1].any()
    assert bad[2, :4].all() and not bad[2, 4:].any()


def test_repeats_are_equal_bit_for_bit():
    c = case(10, [5000, 900, 3], 32, 8, 128, 64, BF)
    op, a = check(*c)
    for _ in range(3):
        assert torch.equal(a, op(*c[:5]))


def test_beyond_32_bit_offsets():
    """Pools past 2^32 bytes: a request whose pages lie at the far end."""
    pages, pr, Hkv, hd = 600, 4096, 8, 128                  # 5.0 GB a pool
    K = torch.zeros(pages, pr, Hkv, hd, dtype=BF, device="cuda")
    V = torch.zeros(pages, pr, Hkv, hd, dtype=BF, device="cuda")
    table = torch.tensor([[599, 598, 0], [1, 597, 2]], dtype=torch.int32, device="cuda")
    for p in (0, 1, 2, 597, 598, 599):
        K[p].normal_()
        V[p].normal_()
    Q = torch.randn(2, 8, hd, device="cuda").to(BF)
    lens = torch.tensor([4200, 8000], dtype=torch.int32, device="cuda")
    op = taps.PagedDecodeAttention(2, 8, Hkv, hd, 9000, pr)
    got = op(Q, K, V, table, lens)
    small = torch.tensor([[3, 4, 5], [0, 1, 2]], dtype=torch.int32, device="cuda")
    sub = torch.tensor([1, 597, 2, 599, 598, 0], device="cuda")
    assert torch.equal(got, op(Q, K[sub].contiguous(), V[sub].contiguous(), small, lens))


def test_two_graphs_and_streams_do_not_share_scratch():
    """Two captured calls of one object, replayed on two streams at once, with eager calls on a
    third: each has the result of its own inputs."""
    a = case(11, [5000, 64], 32, 8, 128, 64, BF)
    b = case(12, [4000, 4999], 32, 8, 128, 64, BF, max_len=5000)
    op, ra = check(*a)
    op2, rb = check(*b)
    assert op.shape == op2.shape
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    graphs, outs = [], []
    for s, x in ((s1, a), (s2, b)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(op(*x[:5]))
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, g in ((s1, graphs[0]), (s2, graphs[1])):
            with torch.cuda.stream(s):
                g.replay()
        e = op(*a[:5])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], ra) and torch.equal(outs[1], rb) and torch.equal(e, ra)


def test_refuses_wrong_tensors():
    Q, K, V, table, lens, m = case(13, [40, 50], 8, 2, 64, 32, BF)
    op = taps.PagedDecodeAttention(2, 8, 2, 64, m, 32)
    for bad in ((Q[:1], K, V, table, lens), (Q, K[:, :16], V, table, lens),
                (Q, K, V[:-1], table, lens), (Q, K, V, table[0], lens),
                (Q, K, V, table[:, ::2], lens),
                (Q.transpose(1, 2).contiguous().transpose(1, 2), K, V, table, lens)):
        with pytest.raises(ValueError):
            op(*bad)
    for bad in ((Q.float(), K, V, table, lens), (Q, K, V, table.long(), lens),
                (Q, K, V, table, lens.cpu())):
        with pytest.raises(TypeError):
            op(*bad)
    with pytest.raises(taps.TapsError):
        op(Q, K, V, table[:, :1].contiguous(), lens)        # too short for max_len
    with pytest.raises(taps.TapsError):
        taps.PagedDecodeAttention(2, 8, 3, 64, 50, 32)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("batch,lo,hi,Hq,Hkv,hd", [
    (70, 0, 3000, 8, 2, 64), (130, 0, 900, 4, 1, 128), (9, 0, 2200, 34, 1, 64), (300, 1, 400, 2, 1, 64),
    (64, 0, 1024, 16, 8, 64), (5, 3000, 3000, 8, 8, 128),
])
def test_equal_parts_of_ragged_batches(dtype, batch, lo, hi, Hq, Hkv, hd):
    """Parts that end inside requests and span several, empty requests among them; more parts
    than units; batches past 64 requests; one workgroup per request."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(lo, hi + 1, batch)]
    if lo == 0:
        lens[0] = lens[-1] = lens[batch // 2] = lens[batch // 2 + 1] = 0
    check(*case(batch + hi, lens, Hq, Hkv, hd, 64, dtype, max_len=hi + 5))
