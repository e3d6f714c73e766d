"""qk_rope_paged against norm and rotation in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def f64(t):
    return t.double().cpu().numpy()


def inputs(seed, rows, Hq, Hkv, hd, page_rows, dtype, far=40000, fused=True, norm=True, pad=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if fused:   # slices of the projection's rows
        x = (r(rows, (Hq + 2 * Hkv) * hd) * 3).to(dtype)
        q, k, v = x.split([Hq * hd, Hkv * hd, Hkv * hd], dim=1)
        Q, K, V = q.unflatten(1, (Hq, hd)), k.unflatten(1, (Hkv, hd)), v.unflatten(1, (Hkv, hd))
    else:
        Q, K, V = (r(rows, h, hd).to(dtype) for h in (Hq, Hkv, Hkv))
    pages = -(-rows // page_rows) + 2
    slots = torch.randperm(pages * page_rows, generator=g, device="cuda")[:rows]
    if pad:
        slots[::7] = -1
    pos = torch.randint(0, far, (rows,), generator=g, device="cuda", dtype=torch.int32)
    Kp, Vp = (r(pages, page_rows, Hkv, hd).to(dtype) for _ in range(2))
    w = [(1 + 0.3 * r(hd)).to(dtype) if norm else None for _ in range(2)]
    return Q, K, V, pos, slots, Kp, Vp, *w


def check(inp, freq, mscale=1.0, interleaved=False, eps=1e-6, out=None):
    """|error|: the last rounding (half a step); times the pair's |a| + |b| and mscale: the norm
    (12 roundings of the sum of squares, halved by the root, the root's own unit and two products:
    10), the reduced angle and its series (4) and the rotation's products and sum (3), 17 x 2^-24,
    under 2^-19."""
    Q, K, V, pos, slots, Kp, Vp, qw, kw = inp
    dtype, (rows, Hq, hd) = Q.dtype, Q.shape
    Hkv, pr = Kp.shape[2], Kp.shape[1]
    op = taps.PagedQKRope(Hq, Hkv, hd, pr, freq, dtype=taps.BF16 if dtype == BF else taps.FP32,
                          interleaved=interleaved, mscale=mscale, eps=eps)
    h = lambda w: None if w is None else f64(w)  # noqa: E731
    want = oracle.qk_rope_paged(f64(Q), f64(K), f64(V), pos.cpu().numpy(), slots.cpu().numpy(),
                                f64(freq), mscale, interleaved, h(qw), h(kw), eps, f64(Kp), f64(Vp))
    K0, V0 = Kp.clone(), Vp.clone()
    got = op(Q, K, V, pos, slots, Kp, Vp, q_norm=qw, k_norm=kw, out=out)
    torch.cuda.synchronize()
    step = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    for name, a, ref, mag in (("Q", got, want[0], want[3]), ("K", Kp, want[1], want[4])):
        err, lim = np.abs(f64(a) - ref), np.abs(ref) * step + abs(mscale) * mag * 2.0 ** -19
        print(f"{name}: max error {err.max():.3e}, at most {np.max(err / (lim + 1e-300)):.3f} of its bound",
              flush=True)
        assert (err <= lim).all(), name
    assert np.array_equal(f64(Vp), want[2])
    s = slots[(slots >= 0) & (slots < Kp.shape[0] * pr)]
    untouched = torch.ones(Kp.shape[0] * pr, dtype=torch.bool, device="cuda")
    untouched[s] = False
    for a, b in ((Kp, K0), (Vp, V0)):
        assert torch.equal(a.flatten(0, 1)[untouched], b.flatten(0, 1)[untouched])
    return op, got


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd,rot", [(128, 128), (128, 64), (128, 24), (128, 8), (64, 64), (64, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts(dtype, hd, rot, interleaved):
    freq, _ = taps.rope_frequencies(rot, 1e4)
    check(inputs(rot + hd, 37, 6, 2, hd, 32, dtype), freq, interleaved=interleaved)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (32, 8), (5, 1), (64, 8), (7, 7)])
@pytest.mark.parametrize("rows", [1, 3, 200])
@pytest.mark.parametrize("norm", [False, True])
def test_heads_and_rows(Hq, Hkv, rows, norm):
    freq, _ = taps.rope_frequencies(128)
    check(inputs(rows + Hq, rows, Hq, Hkv, 128, 64, BF, norm=norm, fused=Hq != 4, pad=rows > 1), freq)
    freq, _ = taps.rope_frequencies(32)
    check(inputs(rows + Hq, rows, Hq, Hkv, 64, 64, FP, norm=norm, fused=Hq != 5), freq)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_far_positions_and_scalings(scaling):
    """Angles of positions past 2^24 and below 0: fp32 products are off by whole turns there."""
    freq, m = taps.rope_frequencies(64, 5e5, scaling=scaling, factor=8.0, trained_len=8192)
    ref, rm = oracle.rope_frequencies(64, 5e5, scaling, 8.0, 8192)
    assert np.allclose(f64(freq), ref, rtol=1e-13, atol=0) and abs(m - rm) <= 2.0 ** -24 * rm
    inp = list(inputs(5, 64, 4, 2, 64, 32, FP, far=2 ** 31 - 1))
    inp[3][:4] = torch.tensor([0, -1, -(2 ** 31), 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    check(inp, freq, mscale=m)


def test_one_norm_and_large_values():
    freq, _ = taps.rope_frequencies(128)
    inp = list(inputs(8, 40, 8, 2, 128, 32, BF))
    inp[0].mul_(2.0 ** 20)
    inp[1].mul_(2.0 ** -20)
    check([*inp[:7], inp[7], None], freq)
    check([*inp[:7], None, inp[8]], freq, eps=0.0)


def test_zero_rows_and_values_that_do_not_turn():
    """A zero head stays zero (eps > 0); infinities and NaN behind the rotated part stay where
    they are, without a norm."""
    freq, _ = taps.rope_frequencies(32)
    Q, K, V, pos, slots, Kp, Vp, _, _ = inputs(9, 20, 4, 2, 64, 32, FP, norm=False, pad=False)
    Q, K = Q.contiguous(), K.contiguous()
    Q[3], K[5] = 0, 0
    Q[0, 0, 40], Q[1, 1, 63], K[2, 1, 33] = float("inf"), float("nan"), float("-inf")
    op = taps.PagedQKRope(4, 2, 64, 32, freq, dtype=taps.FP32)
    out = op(Q, K, V, pos, slots, Kp, Vp)
    assert torch.equal(out[..., 32:].nan_to_num(7, 8, 9), Q[..., 32:].nan_to_num(7, 8, 9))
    assert torch.isfinite(out[..., :32]).all()
    assert torch.equal(Kp.flatten(0, 1)[slots][..., 32:], K[..., 32:])
    one = torch.ones(64, device="cuda")
    out = op(Q, K, V, pos, slots, Kp, Vp, q_norm=one, k_norm=one)
    assert (out[3] == 0).all() and (Kp.flatten(0, 1)[slots[5]] == 0).all()


def test_slots_outside_the_pool_and_given_output():
    freq, _ = taps.rope_frequencies(128)
    inp = list(inputs(11, 33, 4, 2, 128, 32, BF))
    total = inp[5].shape[0] * 32
    inp[4][1], inp[4][2], inp[4][3] = total, 2 ** 62, -(2 ** 62)
    buf = torch.full((35, 4, 128), 3.0, dtype=BF, device="cuda")
    _, got = check(inp, freq, out=buf[1:34])
    assert got.data_ptr() == buf[1:34].data_ptr() and (buf[0] == 3).all() and (buf[34] == 3).all()


def test_no_rows():
    freq, _ = taps.rope_frequencies(128)
    Q, K, V, pos, slots, Kp, Vp, qw, kw = inputs(1, 2, 4, 2, 128, 32, BF)
    K0 = Kp.clone()
    op = taps.PagedQKRope(4, 2, 128, 32, freq)
    out = op(Q[:0], K[:0], V[:0], pos[:0], slots[:0], Kp, Vp)
    assert out.shape == (0, 4, 128) and torch.equal(Kp, K0)


def test_memory_that_meets_is_refused():
    freq, _ = taps.rope_frequencies(128)
    Q, K, V, pos, slots, Kp, Vp, _, _ = inputs(2, 8, 4, 2, 128, 32, BF, fused=False)
    op = taps.PagedQKRope(4, 2, 128, 32, freq)
    with pytest.raises(taps.TapsError):
        op(Q, K, V, pos, slots, Kp, Vp, out=Q)
    with pytest.raises(taps.TapsError):
        op(Q, Kp.flatten(0, 1)[:8], V, pos, slots, Kp, Vp)
    with pytest.raises(taps.TapsError):
        op(Q, K, V, pos, slots, Kp, Kp)


def test_streams_and_graph_replays():
    freq, _ = taps.rope_frequencies(128)
    Q, K, V, pos, slots, Kp, Vp, qw, kw = inputs(21, 50, 8, 2, 128, 32, BF, fused=False, pad=False)
    op = taps.PagedQKRope(8, 2, 128, 32, freq)
    want = op(Q, K, V, pos, slots, Kp, Vp, qw, kw)
    wK = Kp.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = op(Q, K, V, pos, slots, Kp, Vp, qw, kw)
    torch.cuda.synchronize()
    assert torch.equal(other, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = op(Q, K, V, pos, slots, Kp, Vp, qw, kw)
    for i in range(3):
        Kp.zero_()
        out.zero_()
        Q.add_(0 if i == 0 else 1)   # new values in the same memory
        g.replay()
        torch.cuda.synchronize()
        again_K = Kp.clone()
        eager = op(Q, K, V, pos, slots, Kp, Vp, qw, kw)
        assert torch.equal(out, eager) and torch.equal(again_K, Kp)
        if i == 0:
            assert torch.equal(out, want) and torch.equal(again_K[again_K != 0], wK[again_K != 0])


def test_arguments_are_checked():
    freq, _ = taps.rope_frequencies(128)
    Q, K, V, pos, slots, Kp, Vp, qw, kw = inputs(3, 8, 4, 2, 128, 32, BF)
    op = taps.PagedQKRope(4, 2, 128, 32, freq)
    for bad in ((Q.float(), K, V, pos, slots, Kp, Vp), (Q, K, V, pos.long(), slots, Kp, Vp),
                (Q, K, V, pos, slots.int(), Kp, Vp), (Q, K, V.cpu(), pos, slots, Kp, Vp)):
        with pytest.raises(TypeError):
            op(*bad)
    for bad in ((Q[:, :3], K, V, pos, slots, Kp, Vp), (Q, K[:7], V, pos, slots, Kp, Vp),
                (Q, K, V, pos[:7], slots, Kp, Vp), (Q, K, V, pos, slots[1:], Kp, Vp),
                (Q, K, V, pos, slots, Kp[:, :16], Vp)):
        with pytest.raises(ValueError):
            op(*bad)
    with pytest.raises(ValueError):
        op(Q, K, V, pos, slots, Kp, Vp, q_norm=qw[:64])
    with pytest.raises(TypeError):
        taps.PagedQKRope(4, 2, 128, 32, freq.float())
    with pytest.raises(taps.TapsError):
        taps.PagedQKRope(4, 2, 128, 32, freq[:6])(Q, K, V, pos, slots, Kp, Vp)   # 12 dims
    with pytest.raises(ValueError):
        taps.rope_frequencies(64, scaling="cubic")
    with pytest.raises(taps.TapsError):
        taps.rope_frequencies(63)


def test_pool_rows_past_32_bits():
    """Slots whose bytes lie past 4 GB; the rows beside them stay."""
    freq, _ = taps.rope_frequencies(128)
    Q, K, V, pos, _, _, _, qw, kw = inputs(31, 6, 4, 8, 128, 32, BF, fused=False, pad=False)
    pages = 70000
    far = torch.tensor([pages * 32 - 1, 5, 2 ** 21 + 1, 2 ** 21 - 1, pages * 32 - 3, 2 ** 21 + 99],
                       device="cuda")
    Kp = torch.empty(pages, 32, 8, 128, dtype=BF, device="cuda")
    Vp = torch.empty_like(Kp)
    beside = (far - 1).clamp(min=0)
    Kp.flatten(0, 1)[beside], Vp.flatten(0, 1)[beside] = 3.0, 4.0
    op = taps.PagedQKRope(4, 8, 128, 32, freq)
    out = op(Q, K, V, pos, far, Kp, Vp, qw, kw)
    K1, V1 = Kp[:2].clone(), Vp[:2].clone()
    near = torch.arange(6, device="cuda") * 2 + 1
    want = op(Q, K, V, pos, near, K1, V1, qw, kw)
    assert torch.equal(out, want)
    assert torch.equal(Kp.flatten(0, 1)[far], K1.flatten(0, 1)[near])
    assert torch.equal(Vp.flatten(0, 1)[far], V)
    assert (Kp.flatten(0, 1)[beside] == 3).all() and (Vp.flatten(0, 1)[beside] == 4).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_negative_positions(dtype):
    freq, _ = taps.rope_frequencies(64, 1e4)
    inp = list(inputs(32, 40, 4, 2, 128, 32, dtype))
    inp[3] = torch.arange(-20, 20, dtype=torch.int32, device="cuda") * 1001
    check(inp, freq)
