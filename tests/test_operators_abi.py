"""The serving calls around the round refuse bad arguments on the host (no kernel runs here)."""
import ctypes
import math

import pytest

from paper_2606_00487_amd import _lib

OK, INV, UNS, WS = (_lib.TAPS_OK, _lib.TAPS_ERR_INVALID_ARG, _lib.TAPS_ERR_UNSUPPORTED,
                    _lib.TAPS_ERR_WORKSPACE)
F = 1 << 20    # aligned, never dereferenced: every case stops before a launch


def reserve(lib, **kw):
    a = dict(table=F, max_pages=130, held=F, ctx=F, new=F, batch=4, max_new=64, free=F, n_free=F,
             num_pages=600, page_rows=64, held_out=F + 64, n_free_out=F + 128, short=F, slots=F)
    a.update(kw)
    return lib.kv_reserve_paged(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK),
    (dict(batch=-1), INV),
    (dict(batch=4097), UNS),
    (dict(max_pages=0), INV),
    (dict(max_new=-1), INV),
    (dict(max_new=(1 << 27) + 1), UNS),
    (dict(num_pages=0), INV),
    (dict(page_rows=48), INV),
    (dict(page_rows=16), INV),
    (dict(page_rows=8192), INV),
    (dict(max_pages=(1 << 24) + 1), UNS),                  # more than 2^30 rows a request
    (dict(num_pages=(1 << 26)), UNS),                      # pool rows past 32 bits
    (dict(held_out=F), INV),                               # the held_pages array
    (dict(n_free_out=F), INV),
    (dict(slots=F + 4), INV),
    (dict(free=F + 2), INV),
] + [({k: None}, INV) for k in ("table", "held", "ctx", "new", "free", "n_free", "held_out",
                               "n_free_out", "short")])
def test_reserve_refuses(lib, kw, status):
    assert reserve(lib, **kw) == status


def append(lib, **kw):
    a = dict(K=F, V=F, ks=1024, vs=6144, slots=F, rows=8, Hkv=8, hd=128, dtype=0, Kp=F, Vp=F,
             num_pages=10, page_rows=64)
    a.update(kw)
    return lib.kv_append_paged(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), OK),
    (dict(rows=-1), INV),
    (dict(Hkv=0), INV),
    (dict(hd=96), UNS),
    (dict(dtype=2), INV),
    (dict(page_rows=33), INV),
    (dict(num_pages=0), INV),
    (dict(num_pages=1 << 26), UNS),
    (dict(ks=1023), INV),                                  # shorter than a row
    (dict(ks=1028), INV),                                  # not a multiple of 16 bytes
    (dict(vs=1 << 32), UNS),
    (dict(K=F + 8), INV),
    (dict(Vp=F + 8), INV),
    (dict(slots=F + 4), INV),
] + [({k: None}, INV) for k in ("K", "V", "slots", "Kp", "Vp")])
def test_append_refuses(lib, kw, status):
    assert append(lib, **kw) == status


def decode(lib, **kw):
    a = dict(Q=F, qs=4096, K=F, V=F, num_pages=600, page_rows=64, table=F, max_pages=128, len=F,
             batch=4, Hq=32, Hkv=8, hd=128, max_len=8192, dtype=0, scale=0.088, O=F, ws=F,
             ws_bytes=1 << 40)
    a.update(kw)
    return lib.decode_attn_paged(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK),
    (dict(batch=-1), INV),
    (dict(Hq=30), INV),
    (dict(Hkv=0), INV),
    (dict(hd=96), UNS),
    (dict(dtype=3), INV),
    (dict(scale=0.0), INV),
    (dict(scale=math.nan), INV),
    (dict(page_rows=100), INV),
    (dict(num_pages=0), INV),
    (dict(num_pages=1 << 26), UNS),
    (dict(max_pages=127), INV),                            # 127 * 64 < 8192
    (dict(max_len=-1), INV),
    (dict(max_len=(1 << 30) + 1), UNS),
    (dict(batch=8192, Hkv=8), UNS),                        # batch * Hkv past 65535
    (dict(qs=4095), INV),
    (dict(qs=4100), INV),
    (dict(Q=F + 8), INV),
    (dict(O=F + 8), INV),
    (dict(len=F + 2), INV),
    (dict(ws=None), WS),
    (dict(ws=F + 8), WS),
    (dict(ws_bytes=0), WS),
] + [({k: None}, INV) for k in ("Q", "K", "V", "table", "len", "O")])
def test_decode_refuses(lib, kw, status):
    assert decode(lib, **kw) == status


def test_decode_workspace(lib):
    f = lib.decode_attn_paged_workspace_bytes
    a = f(4, 32, 8, 128, 8192, 64, 0)
    assert a > 0 and a == f(4, 32, 8, 128, 8192, 64, 0)
    assert decode(lib, ws_bytes=a - 1) == WS
    assert f(4, 32, 8, 128, 100, 64, 0) == 0               # one split
    assert f(0, 32, 8, 128, 8192, 64, 0) == 0
    assert f(4, 32, 8, 96, 8192, 64, 0) == 0


def sample(lib, **kw):
    a = dict(x=F, stride=151936, batch=2, budget=64, vocab=151936, dtype=0, n=F, s=None, u=F,
             tok=F, pr=F, ws=F, ws_bytes=1 << 40)
    st = kw.pop("settings", _lib.Sampling(F, F, F, F))
    a.update(kw)
    if "s" not in kw:
        a["s"] = ctypes.byref(st)
    return lib.taps_sample(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), OK),
    (dict(batch=-1), INV),
    (dict(budget=0), INV),
    (dict(budget=513), UNS),
    (dict(vocab=0), INV),
    (dict(stride=151935), INV),
    (dict(vocab=(1 << 20) + 1, stride=1 << 21), UNS),
    (dict(stride=1 << 32), UNS),
    (dict(dtype=2), INV),
    (dict(batch=1 << 15), UNS),                            # 2^21 rows
    (dict(x=F + 8), INV),
    (dict(u=F + 2), INV),
    (dict(settings=_lib.Sampling(F, F + 1, F, F)), INV),
] + [({k: None}, INV) for k in ("x", "s", "u", "tok")])
def test_sample_refuses(lib, kw, status):
    assert sample(lib, **kw) == status
