"""chunk_attn_paged against attention in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def case(seed, lens, Hq, Hkv, hd, page_rows, dtype, window=0, pad=0, lead=0, scale_q=1.0, extra=3):
    """lens: (new tokens, cache rows) per request.  Pages in random order; rows that no token sees
    are NaN, entries of the block table that none needs are junk."""
    rng = np.random.default_rng(seed)
    B, max_len = len(lens), max(max(k for _, k in lens), 1)
    need = [-(-k // page_rows) for _, k in lens]
    pages, width = sum(need) + extra, -(-max_len // page_rows) + 1
    ids = rng.permutation(pages)
    table = rng.choice([-5, 2 ** 31 - 1, pages], (B, width))
    own = torch.zeros(pages, page_rows, dtype=torch.bool)
    at = 0
    for b, m in enumerate(need):
        n, k = lens[b]
        low = max(0, k - n - window + 1) if window else 0
        for j in range(m):
            if n > 0 and (j + 1) * page_rows > low:
                table[b, j] = ids[at + j]
                own[ids[at + j], max(0, low - j * page_rows):max(0, k - j * page_rows)] = True
        at += m
    start = np.cumsum([lead] + [n for n, _ in lens])
    rows = int(start[-1]) + pad
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    Q = (r(rows, Hq, hd) * scale_q).to(dtype)
    K, V = r(pages, page_rows, Hkv, hd).to(dtype), r(pages, page_rows, Hkv, hd).to(dtype)
    K[~own], V[~own] = float("nan"), float("nan")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return Q, K, V, i32(table), i32(start), i32([k for _, k in lens]), max_len


def bound(O, A, D, N, hd, scale, dtype):
    """|error| of the outputs: the last rounding (half a step), and times A = sum of the weights
    times |v|: the scores' error (hd products and sums of q k, the scale's and the exponent's own
    roundings, an exponential good to two units), twice since it enters the weights and their sum;
    a rounding per key in the sums of weights and of outputs; bf16: the weights' rounding to bf16,
    half a step of each."""
    n = N[:, None, None].astype(np.float64)
    score = scale * D[..., None] * (hd + 6) * 2.0 ** -24 + 64 * 2.0 ** -24
    rel = 2 * score + 2 * (n + 64) * 2.0 ** -24 + (2.0 ** -8 if dtype == BF else 0.0)
    return np.abs(O) * (2.0 ** -8 if dtype == BF else 2.0 ** -24) + A * rel + 1e-30


def call(Q, K, V, table, start, kv, max_len, window=0, scale=None, out=None):
    op = taps.PagedChunkAttention(len(kv), Q.shape[0], Q.shape[1], K.shape[2], Q.shape[2], max_len,
                                  K.shape[1], dtype=taps.BF16 if Q.dtype == BF else taps.FP32,
                                  scale=scale, window=window)
    return op, op(Q, K, V, table, start, kv, out=out)


def check(inp, window=0, scale=None):
    Q, K, V, table, start, kv, max_len = inp
    out = torch.full(Q.shape, 7.0, dtype=Q.dtype, device="cuda")
    op, O = call(*inp, window=window, scale=scale, out=out)
    h = lambda x: x.double().cpu().numpy()  # noqa: E731
    with np.errstate(invalid="ignore"):
        ref, A, D, N = oracle.chunk_attention_paged(h(Q), h(K), h(V), table.cpu().numpy(),
                                                    start.cpu().numpy(),
                                                    kv.clamp(0, max_len).cpu().numpy(), op.scale,
                                                    window)
    got = h(O)
    none = np.isnan(ref).all(axis=(1, 2))
    assert (got[none] == 7).all()                       # rows of no request stay
    got, ref, A, D, N = got[~none], ref[~none], A[~none], D[~none], N[~none]
    assert np.isfinite(got).all()
    err, lim = np.abs(got - ref), bound(ref, A, D, N, Q.shape[2], op.scale, Q.dtype)
    if err.size:
        print(f"max error {err.max():.3e}, at most {np.max(err / lim):.3f} of its bound", flush=True)
    assert (err <= lim).all()
    return op, O


SHORT = [(1, 1), (2, 2), (0, 5), (31, 31), (32, 32), (33, 40), (1, 64), (5, 65), (64, 64), (65, 127),
         (3, 128), (0, 0), (17, 129)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (10, 2), (16, 1), (33, 3)])
def test_lengths_and_head_layouts(dtype, hd, Hq, Hkv):
    check(case(Hq + hd, SHORT, Hq, Hkv, hd, 32, dtype))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 1000])
@pytest.mark.parametrize("hd", [64, 128])
def test_windows(dtype, window, hd):
    check(case(window, [(1, 400), (300, 300), (70, 500), (130, 131), (2, 2), (40, 37)], 6, 2, hd, 64,
               dtype, window=window), window=window)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("page_rows", [32, 64, 256, 4096])
def test_pages(dtype, page_rows):
    check(case(page_rows, [(100, 700), (1, 4100), (333, 333)], 4, 2, 128, page_rows, dtype))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens", [[(16, 5000)], [(1, 6000), (1, 3), (200, 2500)], [(1, 4097)],
                                  [(257, 1000), (3, 9000)], [(700, 2400)]])
def test_keys_cut_over_workgroups(dtype, hd, lens):
    check(case(len(lens), lens, 8, 2, hd, 64, dtype))
    check(case(len(lens), lens, 3, 1, hd, 64, dtype, window=1500), window=1500)


def test_many_requests():
    """More requests than a wave has lanes; empty ones among them."""
    rng = np.random.default_rng(3)
    lens = [(int(n), int(n + c)) for n, c in zip(rng.integers(0, 40, 150), rng.integers(0, 300, 150))]
    check(case(4, lens, 4, 2, 64, 32, BF, pad=5, lead=3))
    check(case(4, lens, 4, 2, 64, 32, FP, pad=5, lead=3))
    lens[100] = (9, 12000)
    check(case(5, lens, 4, 2, 128, 32, BF))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_tokens_that_see_no_row(dtype):
    """Fewer cache rows than new tokens: the first ones get zeros."""
    _, O = check(case(6, [(50, 20), (10, 0), (300, 1), (5, 5)], 4, 2, 128, 32, dtype))
    assert (O[:30] == 0).all() and (O[50:60] == 0).all() and (O[60:359] == 0).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_outside_the_requests_and_lengths_past_the_bound(dtype):
    inp = list(case(7, [(20, 90), (33, 33)], 4, 2, 128, 32, dtype, pad=70, lead=11))
    check(inp)
    inp[5] = inp[5].clone()
    Q, K, V, table, start, kv, max_len = inp
    inp[5][1] = -4                                       # counts as 0
    check(inp)


@pytest.mark.parametrize("dtype,hd", [(BF, 128), (BF, 64), (FP, 128)])
def test_large_scores(dtype, hd):
    """A few keys hold all the weight, the reference maximum moves often."""
    check(case(8, [(150, 900), (1, 2000)], 4, 1, hd, 64, dtype, scale_q=12.0))
    check(case(9, [(150, 900)], 4, 1, hd, 64, dtype), scale=1e-4)


def test_query_rows_apart_and_any_order_of_pages():
    inp = list(case(10, [(40, 300), (70, 70)], 4, 2, 128, 64, BF))
    wide = torch.full((110, 9, 128), float("nan"), dtype=BF, device="cuda")
    wide[:, 2:6] = inp[0]
    _, a = call(*inp)
    inp[0] = wide[:, 2:6]
    _, b = check(inp)
    assert torch.equal(a, b)


def test_one_token_like_decode():
    lens = [(1, k) for k in (1, 33, 500, 2000)]
    inp = case(11, lens, 8, 2, 128, 64, FP)
    _, O = check(inp)
    dec = taps.PagedDecodeAttention(4, 8, 2, 128, inp[6], 64, dtype=taps.FP32)
    assert torch.allclose(O, dec(inp[0], *inp[1:4], inp[5]), rtol=0, atol=1e-5)


def test_a_prompt_in_chunks_equals_the_whole():
    """The same prompt in one call and in ragged chunks, each over the rows before it."""
    whole = case(12, [(777, 777)], 8, 2, 128, 64, FP)
    Q, K, V, table, _, _, max_len = whole
    _, O = call(*whole)
    at, parts = 0, []
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for n in (1, 63, 200, 513):
        parts.append(call(Q[at:at + n], K, V, table, i32([0, n]), i32([at + n]), max_len)[1])
        at += n
    assert torch.allclose(torch.cat(parts), O, rtol=0, atol=2e-6)


def test_pool_rows_past_32_bits():
    """Pages whose bytes lie past 4 GB."""
    pages, pr, Hkv, hd = 70000, 32, 8, 128
    g = torch.Generator(device="cuda").manual_seed(13)
    K = torch.empty(pages, pr, Hkv, hd, dtype=BF, device="cuda")
    V = torch.empty_like(K)
    ids = torch.tensor([[69999, 3, 69998, 66000]], dtype=torch.int32, device="cuda")
    for p in ids[0].tolist():
        K[p] = torch.randn(pr, Hkv, hd, generator=g, device="cuda").to(BF)
        V[p] = torch.randn(pr, Hkv, hd, generator=g, device="cuda").to(BF)
    Q = torch.randn(50, 16, hd, generator=g, device="cuda").to(BF)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    small = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    _, far = call(Q, K, V, ids, i32([0, 50]), i32([120]), 128)
    _, near = check((Q, K[ids[0].long()], V[ids[0].long()], small, i32([0, 50]), i32([120]), 128))
    assert torch.equal(far, near)


def test_refuses_output_in_the_queries_memory():
    inp = case(14, [(8, 8)], 4, 2, 128, 32, BF)
    with pytest.raises(taps.TapsError):
        call(*inp, out=inp[0])
    with pytest.raises(ValueError):
        taps.PagedChunkAttention(1, 7, 4, 2, 128, 8, 32)(inp[0], *inp[1:6])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_same_bits_on_streams_and_in_graphs(dtype):
    inp = case(15, [(60, 3000), (1, 700), (300, 310)], 8, 2, 128, 64, dtype)
    op, want = call(*inp)
    Q, K, V, table, start, kv, _ = inp
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for s in streams:                                    # calls that overlap
        with torch.cuda.stream(s):
            outs += [op(Q, K, V, table, start, kv) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graphs = []
    for _ in range(2):                                   # two graphs, each with scratch of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = op(Q, K, V, table, start, kv)
        graphs.append((g, o))
    for i in range(3):
        kv.copy_(torch.tensor([3000 - 17 * i, 700 - i, 310 - 100 * i], device="cuda"))
        eager = op(Q, K, V, table, start, kv)
        for g, o in graphs:
            o.zero_()
            g.replay()
        torch.cuda.synchronize()
        for _, o in graphs:
            assert torch.equal(o, eager)


@pytest.mark.parametrize("hd,Hq,Hkv,n", [(128, 20, 4, 1700), (64, 16, 2, 2100)])
def test_whole_prompts(hd, Hq, Hkv, n):
    """The tiles of long prompts, their keys not cut."""
    check(case(16, [(n, n)], Hq, Hkv, hd, 128, BF))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_starts_outside_the_rows_are_clamped(dtype):
    Q, K, V, table, start, kv, max_len = case(17, [(20, 90), (43, 100)], 4, 2, 128, 32, dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    _, want = call(Q, K, V, table, i32([0, 20, 63]), kv, max_len)
    _, got = call(Q, K, V, table, i32([-7, 20, 2 ** 31 - 1]), kv, max_len)
    assert torch.equal(got, want)
    out = torch.full_like(Q, 7.0)
    call(Q, K, V, table, i32([2 ** 31 - 1, 5, -(2 ** 31)]), kv, max_len, out=out)
    assert (out == 7).all()                              # decreasing: no request has a row


def test_lengths_past_the_bound_and_pages_outside_the_pool():
    """kv_len past max_len counts as max_len; page ids are clamped: any values, but no fault."""
    Q, K, V, table, start, kv, max_len = case(18, [(20, 200), (64, 64)], 4, 2, 128, 32, BF)
    kv2 = kv.clone()
    kv2[0] = 2 ** 31 - 1
    assert torch.equal(call(Q, K, V, table, start, kv2, 200)[1], call(Q, K, V, table, start, kv, 200)[1])
    wild = torch.where(torch.arange(table.shape[1], device="cuda") % 2 == 0, table, -(2 ** 31))
    call(Q, K, V, wild.int(), start, kv, max_len)
    call(Q, K, V, torch.full_like(table, 2 ** 31 - 1), start, kv, max_len)
    torch.cuda.synchronize()


def test_arguments_are_checked():
    Q, K, V, table, start, kv, max_len = case(19, [(8, 8)], 4, 2, 128, 32, BF)
    op = taps.PagedChunkAttention(1, 8, 4, 2, 128, max_len, 32)
    for bad in ((Q.float(), K, V, table, start, kv), (Q.cpu(), K, V, table, start, kv),
                (Q, K, V, table, start.long(), kv), (Q, K.float(), V, table, start, kv)):
        with pytest.raises(TypeError):
            op(*bad)
    for bad in ((Q[:, :3], K, V, table, start, kv), (Q, K, V[1:], table, start, kv),
                (Q, K, V, table[0], start, kv), (Q, K, V, table, start[:1], kv),
                (Q, K, V, table, start, start), (Q.transpose(0, 1), K, V, table, start, kv),
                (Q, K.transpose(0, 1), V, table, start, kv)):
        with pytest.raises(ValueError):
            op(*bad)
    assert op(Q[:0], K, V, table, start * 0, kv).shape == (0, 4, 128)


def wider(inp, max_len):
    """The same requests under a larger bound of their lengths; the table's new entries are junk."""
    Q, K, V, table, start, kv, _ = inp
    more = -(-max_len // K.shape[1]) - table.shape[1]
    junk = torch.full((table.shape[0], max(more, 0)), -9, dtype=torch.int32, device="cuda")
    return Q, K, V, torch.cat([table, junk], 1).contiguous(), start, kv, max_len


@pytest.mark.parametrize("Hq,Hkv,n,bound_of_len", [(40, 8, 1638, 2048), (40, 8, 1639, 2048),
                                                   (8, 2, 600, 2048), (8, 2, 600, 2049)])
def test_prompts_at_the_borders_of_the_tile_sizes(Hq, Hkv, n, bound_of_len):
    check(wider(case(20, [(n, n)], Hq, Hkv, 128, 64, BF), bound_of_len))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,kv", [(256, 768), (256, 769), (256, 1030), (257, 1024), (257, 1025),
                                  (257, 1500)])
def test_few_and_many_tiles_at_the_borders_of_a_cut(hd, n, kv):
    """8192 and 8224 query rows of all heads; caches that are just not, or just, cut."""
    check(case(21, [(n, kv)], 32, 8, hd, 64, BF))


def test_ragged_batch_in_many_pieces_of_heads_of_64():
    check(case(22, [(300, 4000), (1, 9000), (900, 900), (0, 50), (17, 3000)], 8, 2, 64, 64, BF))
    check(case(23, [(300, 4000), (1, 9000), (900, 900), (0, 50), (17, 3000)], 40, 20, 64, 64, BF))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
def test_scratch_that_holds_nan(dtype, hd):
    """Every part that the second kernel adds was written by the first."""
    Q, K, V, table, start, kv, max_len = case(24, [(40, 5000), (300, 2000), (2, 90), (0, 4000)], 6,
                                              2, hd, 64, dtype)
    op, want = call(Q, K, V, table, start, kv, max_len)
    n = op._ws_bytes(Q.shape[0])
    assert n > 0
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    O = torch.full_like(want, 7.0)
    st = op.lib.chunk_attn_paged(
        Q.data_ptr(), Q.stride(0), K.data_ptr(), V.data_ptr(), K.shape[0], 64, table.data_ptr(),
        table.shape[1], start.data_ptr(), kv.data_ptr(), len(kv), Q.shape[0], 6, 2, hd, max_len, 0,
        taps.BF16 if dtype == BF else taps.FP32, op.scale, O.data_ptr(), ws.data_ptr(), n,
        torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(O, want)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_values_that_are_not_finite_stay_in_their_request(dtype):
    Q, K, V, table, start, kv, max_len = case(25, [(20, 900), (64, 64), (3, 2000), (100, 100)], 4, 2,
                                              128, 32, dtype)
    _, want = call(Q, K, V, table, start, kv, max_len)
    V[table[0, 3].long(), 5, 1, 7] = float("nan")
    V[table[0, 4].long(), 9, 0] = float("inf")
    K[table[2, 0].long(), 3, 0] = float("nan")
    K[table[2, 30].long(), 3, 1] = float("-inf")
    _, got = call(Q, K, V, table, start, kv, max_len)
    assert torch.equal(got[20:84], want[20:84]) and torch.equal(got[87:], want[87:])
    assert torch.isnan(got[:20, 2:, 7]).all() and not torch.isfinite(got[:20, :2]).any()
    assert torch.isnan(got[84:87, :2]).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_queries_that_are_not_finite_stay_in_their_row(dtype):
    Q, K, V, table, start, kv, max_len = case(26, [(20, 900), (64, 64)], 4, 2, 64, 32, dtype)
    _, want = call(Q, K, V, table, start, kv, max_len)
    Q[3, 1, 5], Q[40, 2] = float("nan"), float("inf")
    _, got = call(Q, K, V, table, start, kv, max_len)
    other = torch.ones(84, 4, dtype=torch.bool, device="cuda")
    other[3, 1] = other[40, 2] = False
    assert torch.equal(got[other], want[other]) and torch.isnan(got[3, 1]).all()


def test_requests_with_a_common_beginning():
    """Pages in several tables: the same as copies of them."""
    Q, K, V, table, start, kv, max_len = case(27, [(30, 400), (70, 300)], 4, 2, 128, 32, BF)
    table[1, :6] = table[0, :6]
    _, shared = check((Q, K, V, table, start, kv, max_len))
    K2, V2 = torch.cat([K, K[table[0, :6].long()]]), torch.cat([V, V[table[0, :6].long()]])
    table[1, :6] = torch.arange(K.shape[0], K.shape[0] + 6, device="cuda")
    _, copied = call(Q, K2, V2, table, start, kv, max_len)
    assert torch.equal(shared, copied)


def test_refuses_output_in_the_pools():
    Q, K, V, table, start, kv, max_len = case(28, [(8, 8)], 4, 2, 128, 32, BF)
    for pool in (K, V):
        with pytest.raises(taps.TapsError):
            call(Q, K, V, table, start, kv, max_len, out=pool.view(-1)[:8 * 4 * 128].view(8, 4, 128))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B", [256, 257, 1025, 4100])
def test_more_requests_than_are_added_up_by_every_workgroup(dtype, B):
    """Empty ones among them, and some that are cut."""
    rng = np.random.default_rng(B)
    n = rng.integers(0, 5, B)
    lens = [(int(a), int(a + c)) for a, c in zip(n, rng.integers(0, 60, B))]
    check(case(29, lens, 4, 2, 64, 32, dtype, pad=3, lead=2))
    lens[200], lens[B - 2], lens[B - 1] = (9, 9000), (70, 7000), (0, 0)
    check(case(30, lens, 4, 2, 128, 32, dtype))


def test_index_scratch_that_holds_nan_and_graphs():
    rng = np.random.default_rng(1)
    lens = [(int(a), int(a + 30)) for a in rng.integers(0, 4, 300)]
    Q, K, V, table, start, kv, max_len = case(31, lens, 4, 2, 64, 32, BF)
    op, want = call(Q, K, V, table, start, kv, max_len)
    ws = torch.full((op._ws_bytes(Q.shape[0]),), 0xFF, dtype=torch.uint8, device="cuda")
    del ws                                     # torch's allocator hands the same memory out again
    assert torch.equal(call(Q, K, V, table, start, kv, max_len)[1], want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = op(Q, K, V, table, start, kv)
    for i in range(3):
        out.zero_()
        Q.neg_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, op(Q, K, V, table, start, kv))


def test_many_requests_whose_starts_decrease():
    """Rows that several requests name hold any of theirs; nothing else is written."""
    Q, K, V, table, start, kv, max_len = case(32, [(2, 40)] * 300, 4, 2, 64, 32, BF, pad=4)
    odd = start.clone()
    odd[1::2] = 0
    buf = torch.full((606, 4, 64), 7.0, dtype=BF, device="cuda")
    call(Q, K, V, table, odd, kv, max_len, out=buf[1:605])
    torch.cuda.synchronize()
    assert (buf[0] == 7).all() and (buf[601:] == 7).all()


@pytest.mark.parametrize("n,kv,bound_of_len", [(1168, 1168, 1168), (1172, 1172, 1172), (600, 600, 2560),
                                               (600, 600, 2561), (16, 3000, 3000), (17, 3000, 3000),
                                               (1300, 2500, 2560)])
def test_one_request_at_the_borders_of_pairs(n, kv, bound_of_len):
    """Tiles alone and two workgroups a CU, whole and cut."""
    check(wider(case(33, [(n, kv)], 32, 8, 128, 64, BF), bound_of_len))


@pytest.mark.parametrize("B", [15, 16, 37, 38])
def test_single_tokens_at_the_borders_of_pairs(B):
    rng = np.random.default_rng(B)
    lens = [(1, int(k)) for k in rng.integers(1, 3000, B)]
    lens[3] = (1, 2700)
    check(case(34, lens, 32, 8, 128, 64, BF))
    check(case(35, [(1, min(k, 900)) for _, k in lens], 32, 8, 128, 64, BF))


def test_ragged_prompts_in_pairs():
    rng = np.random.default_rng(5)
    lens = [(int(n), int(n)) for n in rng.integers(1, 700, 12)]
    check(case(36, lens, 16, 4, 128, 32, BF, lead=1, pad=2))
    check(case(37, lens, 16, 4, 128, 32, BF, window=100), window=100)
