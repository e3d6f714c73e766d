"""The calls of a prompt refuse bad arguments on the host (no kernel runs here)."""
import ctypes
import math

import pytest

from paper_2606_00487_amd import _lib

OK, INV, UNS, WS = (_lib.TAPS_OK, _lib.TAPS_ERR_INVALID_ARG, _lib.TAPS_ERR_UNSUPPORTED,
                    _lib.TAPS_ERR_WORKSPACE)
F = 1 << 40    # aligned, never dereferenced: every case stops before a launch
GB = 1 << 32   # memory of its own


def frequencies(lib, rot=64, theta=1e6, scaling=0, factor=1.0, trained=1, out=True, m=True):
    f, ms = (ctypes.c_double * 2048)(), ctypes.c_float()
    st = lib.taps_rope_frequencies(rot, theta, scaling, factor, trained, f if out else None,
                                   ctypes.byref(ms) if m else None)
    return st


@pytest.mark.parametrize("kw,status", [
    ({}, OK), (dict(rot=2), OK), (dict(rot=4096), OK), (dict(rot=0), INV), (dict(rot=63), INV),
    (dict(rot=4098), INV), (dict(theta=1.0), INV), (dict(theta=math.inf), INV),
    (dict(theta=math.nan), INV), (dict(scaling=4), INV), (dict(scaling=-1), INV),
    (dict(scaling=1, factor=0.5), INV), (dict(scaling=1, factor=math.nan), INV),
    (dict(scaling=0, factor=math.nan), OK), (dict(scaling=3, factor=2.0, trained=0), INV),
    (dict(scaling=2, factor=2.0, rot=2), INV), (dict(scaling=2, factor=1e308, rot=4), INV),
    (dict(out=False), INV), (dict(m=False), INV),
])
def test_frequencies_refuse(lib, kw, status):
    assert frequencies(lib, **kw) == status


def rope(lib, freq=F, qn=F, kn=F, eps=1e-6, mscale=1.0, rot=128, il=0, null=False, **kw):
    a = dict(Q=F + GB, K=F + 2 * GB, V=F + 3 * GB, qs=4096, ks=1024, vs=1024, pos=F, slots=F,
             rows=8, Hq=32, Hkv=8, hd=128, dtype=0)
    b = dict(Qo=F + 4 * GB, Kp=F + 5 * GB, Vp=F + 6 * GB, num_pages=10, page_rows=64)
    for d in (a, b):
        d.update({k: v for k, v in kw.items() if k in d})
    st = _lib.Rope(freq, qn, kn, eps, mscale, rot, il)
    return lib.qk_rope_paged(*a.values(), None if null else ctypes.byref(st), *b.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), OK), (dict(rows=0, Q=None, freq=None), OK), (dict(rows=-1), INV),
    (dict(Hq=0), INV), (dict(Hkv=0), INV), (dict(hd=96), UNS), (dict(dtype=2), INV),
    (dict(page_rows=48), INV), (dict(num_pages=0), INV), (dict(num_pages=1 << 26), UNS),
    (dict(rot=0), INV), (dict(rot=12), INV), (dict(rot=136), INV), (dict(il=2), INV),
    (dict(eps=-1.0), INV), (dict(eps=math.nan), INV), (dict(mscale=math.inf), INV),
    (dict(qs=4095), INV), (dict(qs=4100), INV), (dict(ks=1023), INV), (dict(vs=1 << 32), UNS),
    (dict(Q=F + GB + 8), INV), (dict(Kp=F + 5 * GB + 8), INV), (dict(qn=F + 8), INV),
    (dict(slots=F + 4), INV), (dict(pos=F + 2), INV), (dict(freq=F + 4), INV),
    (dict(Hq=1 << 16), UNS),
    (dict(Qo=F + GB), INV),                                # the queries' own memory
    (dict(Qo=F + GB + 8 * 4096 * 2 - 16), INV),            # its last 16 bytes
    (dict(Kp=F + 2 * GB), INV), (dict(Vp=F + 5 * GB + 16), INV), (dict(Qo=F + 6 * GB), INV),
    (dict(null=True), INV),
] + [({k: None}, INV) for k in ("Q", "K", "V", "pos", "slots", "freq", "Qo", "Kp", "Vp")])
def test_rope_refuses(lib, kw, status):
    assert rope(lib, **kw) == status


def chunk(lib, **kw):
    a = dict(Q=F, qs=4096, K=F + GB, V=F + 2 * GB, num_pages=600, page_rows=64, table=F,
             max_pages=128, start=F, len=F, batch=4, rows=100, Hq=32, Hkv=8, hd=128, max_len=8192,
             window=0, dtype=0, scale=0.088, O=F + 3 * GB, ws=F, ws_bytes=1 << 40)
    a.update(kw)
    return lib.chunk_attn_paged(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK), (dict(rows=0), OK), (dict(batch=-1), INV), (dict(rows=-1), INV),
    (dict(Hq=0), INV), (dict(Hq=33), INV), (dict(Hkv=0), INV), (dict(hd=96), UNS),
    (dict(dtype=3), INV), (dict(page_rows=16), INV), (dict(page_rows=8192), INV),
    (dict(max_len=-1), INV), (dict(max_len=8193), INV), (dict(max_len=(1 << 30) + 1), UNS),
    (dict(window=-1), INV), (dict(window=(1 << 30) + 1), UNS), (dict(scale=0.0), INV),
    (dict(scale=math.nan), INV), (dict(num_pages=0), INV), (dict(num_pages=1 << 26), UNS),
    (dict(max_pages=0), INV), (dict(qs=4088), INV), (dict(qs=4100), INV), (dict(qs=1 << 32), UNS),
    (dict(rows=1 << 26), UNS), (dict(batch=(1 << 20) + 1), UNS), (dict(Hq=65536, qs=65536 * 128), UNS),
    (dict(Q=F + 8), INV), (dict(O=F + 3 * GB + 8), INV), (dict(table=F + 2), INV),
    (dict(start=F + 1), INV), (dict(len=F + 3), INV), (dict(O=F), INV), (dict(O=F + 16), INV),
    (dict(ws=None), WS), (dict(ws_bytes=1000), WS), (dict(ws=F + 8), WS),
] + [({k: None}, INV) for k in ("Q", "K", "V", "table", "start", "len", "O")])
def test_chunk_refuses(lib, kw, status):
    assert chunk(lib, **kw) == status


def test_chunk_workspace_is_bounded_and_none_for_short_caches(lib):
    ws = lib.chunk_attn_paged_workspace_bytes
    assert ws(4, 100, 32, 8, 128, 640, 64, 0) == 0         # 640 rows are never cut
    n = ws(4, 100, 32, 8, 128, 8192, 64, 0)
    assert 0 < n <= 512 * 256 * (128 * 4 + 8)
    assert ws(4, 1 << 20, 32, 8, 128, 1 << 20, 64, 0) == n  # by the pieces, not by the rows
    assert ws(4, 100, 32, 8, 96, 8192, 64, 0) == 0 and ws(0, 100, 32, 8, 128, 8192, 64, 0) == 0


def logprobs(lib, **kw):
    a = dict(x=F, stride=1024, batch=2, budget=3, vocab=1000, dtype=0, n=F, tok=F, top=5, lp=F,
             ent=F, rank=F, idx=F, tlp=F, ws=F, ws_bytes=1 << 30)
    a.update(kw)
    return lib.taps_logprobs(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK), (dict(batch=-1), INV), (dict(budget=0), INV), (dict(vocab=0), INV),
    (dict(stride=999), INV), (dict(dtype=2), INV), (dict(budget=513), UNS),
    (dict(vocab=(1 << 20) + 1, stride=1 << 21), UNS), (dict(batch=1 << 20, budget=2), UNS),
    (dict(top=-1), INV), (dict(top=65), UNS), (dict(vocab=4, top=5), INV),
    (dict(x=F + 2), INV), (dict(x=F + 1, vocab=1001), INV), (dict(tok=F + 2), INV),
    (dict(rank=F + 1), INV), (dict(n=F + 2), INV), (dict(idx=F + 2), INV),
    (dict(vocab=100000, stride=100000, ws=None), WS), (dict(vocab=100000, stride=100000, ws=F + 8), WS),
    (dict(vocab=100000, stride=100000, ws_bytes=99), WS),
] + [({k: None}, INV) for k in ("x", "tok", "lp", "ent", "rank", "idx", "tlp")])
def test_logprobs_refuses(lib, kw, status):
    assert logprobs(lib, **kw) == status


def test_logprobs_workspace_is_for_few_rows(lib):
    ws = lib.taps_logprobs_workspace_bytes
    assert ws(4, 512, 151936, 0, 5) == 0 and ws(1, 1, 1000, 0, 5) == 0 and ws(0, 1, 151936, 0, 5) == 0
    assert 0 < ws(1, 1, 151936, 0, 64) <= 16 * (32 + 8 * 64) and ws(1, 1, 151936, 0, 65) == 0


@pytest.mark.parametrize("kw", [dict(O=F + GB), dict(O=F + 2 * GB + 16),
                                dict(O=F + GB - 100 * 4096 * 2 + 16),
                                dict(K=F + 3 * GB - 600 * 64 * 1024 * 2 + 16)])
def test_chunk_refuses_an_output_in_the_pools(lib, kw):
    assert chunk(lib, **kw) == INV


def test_strides_whose_spans_would_pass_64_bits_are_refused(lib):
    assert rope(lib, qs=(1 << 30) + 8) == UNS and chunk(lib, qs=(1 << 30) + 8) == UNS


def test_chunk_scratch_of_many_requests(lib):
    ws = lib.chunk_attn_paged_workspace_bytes
    assert ws(256, 300, 32, 8, 128, 640, 64, 0) == 0
    assert ws(257, 300, 32, 8, 128, 640, 64, 0) == 258 * 16
    kw = dict(batch=257, rows=300, max_len=640)
    assert chunk(lib, ws=None, **kw) == WS and chunk(lib, ws_bytes=258 * 16 - 1, **kw) == WS
    assert chunk(lib, ws=F + 8, **kw) == WS


def test_chunk_refuses_more_workgroups_than_a_launch_holds(lib):
    """Their threads are counted in 32 bits."""
    v = lib.chunk_attn_paged_validate
    assert v(1 << 20, 1 << 20, 32, 8, 128, 4096, 64, 0, 0, 1.0) == UNS
    assert v(1 << 19, 1 << 20, 32, 8, 128, 4096, 64, 0, 0, 1.0) == OK
    assert v(1, 1 << 24, 64, 8, 128, 4096, 64, 0, 0, 1.0) == OK
    assert v(1, 1 << 24, 64, 8, 64, 4096, 64, 0, 1, 1.0) == UNS


def test_chunk_scratch_is_enough_for_fewer_rows(lib):
    ws = lib.chunk_attn_paged_workspace_bytes
    sizes = [1, 2, 16, 33, 63, 64, 65, 255, 256, 257, 300, 640, 1024, 1025, 2048, 5000, 70000]
    for Hq, Hkv, hd, dt in ((32, 8, 128, 0), (16, 2, 64, 0), (5, 1, 128, 0), (64, 64, 128, 0),
                            (32, 8, 128, 1), (4, 2, 64, 1)):
        for batch in (1, 3, 16, 40, 300):
            for max_len in (64, 192, 193, 700, 768, 769, 1000, 1024, 1025, 2560, 2561, 9000, 100000):
                got = [ws(batch, n, Hq, Hkv, hd, max_len, 64, dt) for n in sizes]
                assert got == sorted(got), (Hq, Hkv, hd, dt, batch, max_len, got)
