"""kv_reserve_paged refuses counts that it would write over what it reads: every workgroup reads
all lengths, while others write theirs (host checks; no kernel runs here)."""
import pytest

from paper_2606_00487_amd import _lib

F = 1 << 20    # aligned, never dereferenced: every case stops before a launch
BATCH = 4
IN = dict(held=F, ctx=F + 256, new=F + 512, n_free=F + 768)
OUT = dict(held_out=F + 1024, n_free_out=F + 1280, short=F + 1536)


def reserve(lib, **kw):
    a = dict(table=F + 4096, max_pages=8, held=0, ctx=0, new=0, batch=BATCH, max_new=16, free=F + 8192,
             n_free=0, num_pages=64, page_rows=64, held_out=0, n_free_out=0, short=0, slots=F + 16384)
    a.update(IN, **OUT)
    a.update(kw)
    return lib.kv_reserve_paged(*a.values(), None)


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("name", IN)
def test_refuses_outputs_in_inputs(lib, out, name):
    words = 1 if name == "n_free" else BATCH
    for word in {0, words // 2, words - 1}:                # anywhere in the array
        assert reserve(lib, **{out: IN[name] + 4 * word}) == _lib.TAPS_ERR_INVALID_ARG


@pytest.mark.parametrize("name", IN)
def test_refuses_page_counts_that_run_into_inputs(lib, name):
    assert reserve(lib, held_out=IN[name] - 4 * (BATCH - 1)) == _lib.TAPS_ERR_INVALID_ARG


def test_other_checks_come_first(lib):
    """The arrays that the cases above start from are taken apart from what they change."""
    assert reserve(lib, batch=0) == _lib.TAPS_OK
    assert reserve(lib, batch=4097, short=IN["n_free"]) == _lib.TAPS_ERR_UNSUPPORTED
