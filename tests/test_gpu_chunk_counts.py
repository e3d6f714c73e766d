"""chunk_attn_paged counts its keys: with equal scores and one-hot values each output is the share of
the keys that carry its dim, and a key that is lost, doubled or another's moves one by percents."""
import numpy as np
import pytest
import torch

import paper_2606_00487_amd as taps

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def check(lens, Hq, Hkv, hd, dtype, window=0, max_len=0, page_rows=32, cut=None):
    """Key j of KV head g carries 1 in dim (j + 5 g) mod hd.  Queries are 0, so that every weight is
    exactly 1 and sums are whole numbers; the output rounds the count's product with 1 / n (three
    fp32 roundings) once.  Rows that no token sees are NaN, their table entries junk."""
    rng = np.random.default_rng(len(lens) + hd + window)
    max_len = max(max_len, max(k for _, k in lens), 1)
    need = [-(-k // page_rows) for _, k in lens]
    pages = sum(need) + 2
    ids, at = rng.permutation(pages), 0
    table = np.full((len(lens), -(-max_len // page_rows) + 1), -7)
    V = np.full((pages * page_rows, Hkv, hd), np.nan, dtype=np.float32)
    K = np.full_like(V, np.nan)
    for b, (n, k) in enumerate(lens):
        low = max(0, k - n - window + 1) if window else 0
        j = np.arange(low, k if n else 0)
        page = ids[at:at + need[b]]
        first = low // page_rows
        table[b, first:need[b]] = page[first:]
        at += need[b]
        r = page[j // page_rows] * page_rows + j % page_rows
        K[r] = rng.normal(size=(len(r), Hkv, hd))
        V[r] = 0
        for g in range(Hkv):
            V[r, g, (j + 5 * g) % hd] = 1
    start = np.cumsum([0] + [n for n, _ in lens])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    K, V = (torch.from_numpy(x).cuda().to(dtype).unflatten(0, (pages, page_rows)) for x in (K, V))
    Q = torch.zeros(int(start[-1]), Hq, hd, dtype=dtype, device="cuda")
    op = taps.PagedChunkAttention(len(lens), len(Q), Hq, Hkv, hd, max_len, page_rows, window=window,
                                  dtype=taps.BF16 if dtype == BF else taps.FP32)
    if cut is not None:
        assert (op._ws_bytes(len(Q)) > 0) == cut
    got = op(Q, K, V, i32(table), i32(start), i32([k for _, k in lens])).double().cpu().numpy()
    step = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    for b, (n, k) in enumerate(lens):
        p = k - n + np.arange(n)
        hi = np.maximum(p + 1, 0)[:, None, None]
        lo = np.maximum(p + 1 - window, 0)[:, None, None] if window else np.zeros_like(hi)
        g = (np.arange(Hq) // (Hq // Hkv))[None, :, None]
        res = (np.arange(hd)[None, None, :] - 5 * g) % hd                # j mod hd
        count = (hi - res + hd - 1) // hd - (lo - res + hd - 1) // hd
        ref = count / np.maximum(hi - lo, 1)
        err = np.abs(got[start[b]:start[b + 1]] - ref)
        assert (err <= ref * (step + 3 * 2.0 ** -24)).all(), (b, n, k)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("units", [1, 2, 3, 9, 16, 23, 40])
def test_tiles_and_pieces_of_one_request(dtype, hd, units):
    """Caches of whole key tiles and one key more or less: single tokens, part of a tile of query
    rows, several tiles."""
    for k in (64 * units - 1, 64 * units, 64 * units + 1):
        for n in (1, 16, 33, k):
            check([(n, k)], 8, 2, hd, dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd,n,k,Hq,Hkv", [
    (128, 1, 6000, 8, 2), (128, 16, 6017, 8, 2), (128, 100, 4097, 8, 2), (128, 300, 4095, 8, 2),
    (128, 700, 8129, 4, 1), (128, 2700, 2700, 8, 8), (128, 5, 9000, 16, 1), (64, 1, 6000, 4, 1),
    (64, 16, 6001, 16, 1), (64, 300, 4097, 8, 2), (64, 1500, 3011, 8, 2)])
def test_long_caches(dtype, hd, n, k, Hq, Hkv):
    """Tiles of 256 rows, of 128 with two workgroups a CU, cut and whole."""
    check([(n, k)], Hq, Hkv, hd, dtype, cut=True)
    check([(n, k), (0, 9), (3, 70), (1, 65)], Hq, Hkv, hd, dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window", [1, 63, 64, 65, 129, 1000, 1500])
def test_windows(dtype, hd, window):
    lens = [(1, 4097), (40, 4000), (300, 3001), (2, 2), (70, 64), (128, 191)]
    check(lens, 6, 2, hd, dtype, window=window)
    check(lens, 16, 1, hd, dtype, window=window, max_len=9000)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
def test_many_requests(dtype, hd):
    rng = np.random.default_rng(hd)
    for batch in (40, 100, 300):
        lens = [(int(n), int(n + c)) for n, c in zip(rng.integers(0, 12, batch),
                                                     rng.integers(0, 200, batch))]
        check(lens, 8, 2, hd, dtype, max_len=5000)
        lens[batch // 2] = (7, 4999)
        check(lens, 8, 2, hd, dtype)
