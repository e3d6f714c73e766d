"""kv_reserve_paged and kv_append_paged against the literal simulation."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu


def pool(rng, batch, width, pages, lens, page_rows):
    """Tables whose requests hold the pages of `lens` rows, and the stack of the others."""
    held = np.array([min(-(-n // page_rows), width) for n in lens], np.int32)
    ids = rng.permutation(pages).astype(np.int32)
    table = rng.integers(0, pages, (batch, width)).astype(np.int32)   # stale entries behind held
    at = 0
    for b in range(batch):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.full(pages, -7, np.int32)
    free[:pages - at] = ids[at:]
    return table, held, free, pages - at


def check(table, held, ctx, new, free, n_free, page_rows, max_new, slot_map=True):
    B, width = table.shape
    want = oracle.kv_reserve_paged(table, held, ctx, new, free, n_free, page_rows, max_new)
    d = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    t, f = d(table), d(free)
    res = taps.PagedKVReserve(B, width, len(free), page_rows, max_new, slot_map=slot_map)
    for _ in range(2):     # the call reads nothing that it writes: a second one says the same
        h, nf, sh, slots = res(t, d(held), d(ctx), d(new), f, d([n_free]))
        np.testing.assert_array_equal(t.cpu().numpy(), want[0])
        np.testing.assert_array_equal(h.cpu().numpy(), want[1])
        np.testing.assert_array_equal(f.cpu().numpy(), want[2])
        assert nf.tolist() == [want[3]] and sh.tolist() == [want[4]]
        if slot_map:
            np.testing.assert_array_equal(slots.cpu().numpy(), want[5])
        else:
            assert slots is None
    return want


@pytest.mark.parametrize("batch,page_rows,hi,max_new,spare", [
    (1, 32, 1, 1, 1), (1, 4096, 9000, 4097, 3), (7, 64, 700, 33, 40), (16, 32, 500, 128, 100),
    (300, 64, 900, 70, 900), (1025, 32, 200, 5, 2000), (4096, 32, 100, 2, 4096),
    (5, 128, 2000, 9000, 400),
])
def test_reserve_matches_simulation(batch, page_rows, hi, max_new, spare):
    rng = np.random.default_rng([batch, page_rows, max_new])
    lens = rng.integers(0, hi + 1, batch)
    width = -(-(hi + max_new) // page_rows)
    pages = int(sum(-(-lens // page_rows))) + spare
    table, held, free, nf = pool(rng, batch, width, pages, lens, page_rows)
    new = rng.integers(0, max_new + 1, batch)
    ended = rng.random(batch) < 0.25
    ctx, new = np.where(ended, 0, lens), np.where(ended, 0, new)
    check(table, held, ctx, new, free, nf, page_rows, max_new)
    check(table, held, ctx, new, free, nf, page_rows, max_new, slot_map=False)


@pytest.mark.parametrize("batch,n_free", [(9, 0), (9, 3), (64, 10), (700, 60), (700, 0)])
def test_reserve_when_the_pool_runs_out(batch, n_free):
    """Requests in order until one is short; pages given back in the same call are taken."""
    rng = np.random.default_rng([batch, n_free])
    lens = rng.integers(1, 300, batch)
    table, held, free, nf = pool(rng, batch, 16, int(sum(-(-lens // 32))) + n_free, lens, 32)
    ended = np.arange(batch) % 6 == 5
    ctx = np.where(ended, 0, lens)
    new = np.where(ended, 0, rng.integers(0, 90, batch))
    w = check(table, held, ctx, new, free, nf, 32, 90)
    assert w[4] > 0 or n_free > 3


def test_reserve_odd_counts():
    """Lengths and counts outside their ranges are clamped; rows past the table are short."""
    rng = np.random.default_rng(3)
    table, held, free, nf = pool(rng, 6, 4, 40, [10, 40, 70, 128, 0, 33], 32)
    held = np.array([1, 2, 3, 9, -4, 2], np.int32)        # 9 -> 4, -4 -> 0
    check(table, held, [10, -5, 70, 128, 0, 2 ** 31 - 1], [200, -1, 58, 1, 7, 60], free, nf, 32, 60)
    check(table, held, [0] * 6, [0] * 6, free, 99, 32, 60)          # n_free past the pool
    check(table, held, [1] * 6, [1] * 6, free, -3, 32, 60)
    check(table, held, [1] * 6, [0] * 6, free, nf, 32, 0, slot_map=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,Hkv,hd,page_rows,fused", [
    (1, 1, 64, 32, False), (37, 2, 64, 64, True), (64, 8, 128, 64, True), (513, 3, 128, 32, False),
    (3000, 8, 128, 4096, True),
])
def test_append_matches_simulation(dtype, rows, Hkv, hd, page_rows, fused):
    rng = np.random.default_rng([rows, Hkv, hd])
    g = torch.Generator(device="cuda").manual_seed(rows)
    pages = -(-rows // page_rows) + 2
    slots = rng.permutation(pages * page_rows)[:rows].astype(np.int64)
    slots[rng.random(rows) < 0.1] = rng.choice([-1, -2 ** 62, pages * page_rows, 2 ** 40])
    pk = torch.randn(pages, page_rows, Hkv, hd, generator=g, device="cuda").to(dtype)
    pv = torch.randn(pages, page_rows, Hkv, hd, generator=g, device="cuda").to(dtype)
    if fused:
        f = torch.randn(rows, 4 * Hkv * hd, generator=g, device="cuda").to(dtype)
        k, v = (x.unflatten(1, (Hkv, hd)) for x in f[:, 2 * Hkv * hd:].chunk(2, dim=1))
    else:
        k, v = (torch.randn(rows, Hkv, hd, generator=g, device="cuda").to(dtype) for _ in range(2))
    h = lambda x: x.float().cpu().numpy()  # noqa: E731
    want = oracle.kv_append_paged(h(k), h(v), slots, h(pk), h(pv))
    op = taps.PagedKVAppend(Hkv, hd, page_rows, dtype=taps.BF16 if dtype == torch.bfloat16 else taps.FP32)
    op(k, v, torch.from_numpy(slots).cuda(), pk, pv)
    assert np.array_equal(h(pk), want[0]) and np.array_equal(h(pv), want[1])


def test_append_beyond_32_bit_offsets():
    """A pool whose rows lie past 2^32 bytes: the rows land there, the ones beside them stay."""
    Hkv, hd, pr = 8, 128, 4096
    pages = 600                                             # 600 * 4096 * 2 KB = 5.0 GB a pool
    pk = torch.zeros(pages, pr, Hkv, hd, dtype=torch.bfloat16, device="cuda")
    pv = torch.zeros_like(pk)
    k = torch.randn(3, Hkv, hd, device="cuda").bfloat16()
    slots = torch.tensor([pages * pr - 1, 2 ** 21 + 5, 0], device="cuda")
    taps.PagedKVAppend(Hkv, hd, pr)(k, -k, slots, pk, pv)
    for p, x in ((pk, k), (pv, -k)):
        flat = p.view(-1, Hkv, hd)
        assert torch.equal(flat[slots], x)
        assert int(torch.count_nonzero(flat.abs().amax((1, 2)))) == 3


def test_refuses_wrong_tensors():
    i32 = dict(dtype=torch.int32, device="cuda")
    res = taps.PagedKVReserve(2, 4, 8, 32, 5)
    t, h, f, n = (torch.zeros(s, **i32) for s in ((2, 4), (2,), (8,), (1,)))
    with pytest.raises(ValueError):
        res(t, h, h, h, f[:7], n)
    with pytest.raises(TypeError):
        res(t, h.long(), h, h, f, n)
    with pytest.raises(TypeError):
        res(t.cpu(), h, h, h, f, n)
    op = taps.PagedKVAppend(2, 64, 32)
    p = torch.zeros(3, 32, 2, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        op(k, k[:3], s, p, p.clone())
    with pytest.raises(ValueError):
        op(k.transpose(1, 2).contiguous().transpose(1, 2), k, s, p, p.clone())
    with pytest.raises(TypeError):
        op(k.float(), k, s, p, p.clone())
