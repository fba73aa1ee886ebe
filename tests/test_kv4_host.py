"""The 4-bit key/value cache's host side (no GPU): pool sizes, and calls that are refused before anything is queued."""
import ctypes as C

import pytest
import torch

import kv4_utils as ku
from paper_2604_23467_amd import binding as b


@pytest.mark.parametrize("kv_heads,head_dim,page,pages", [(1, 64, 1, 1), (2, 128, 16, 7), (5, 64, 7, 33), (32, 128, 64, 1000)])
def test_pool_bytes(kv_heads, head_dim, page, pages):
    codes, params = ku.regions(kv_heads, head_dim, page * pages)
    assert b.ll_kv4_pool_bytes(kv_heads, head_dim, page, pages) == 2 * (codes + params)


def test_pool_bytes_of_unsupported_shapes():
    for shape in ((0, 64, 16, 4), (2, 96, 16, 4), (2, 64, 0, 4), (2, 64, 16, 0), (2, 64, 1 << 13, (1 << 13) + 1), (5000, 64, 16, 4)):
        assert b.ll_kv4_pool_bytes(*shape) == 0, shape
    assert b.ll_kv4_pool_bytes(2, 64, 1 << 13, 1 << 13) > 0
    assert b.load().ll_kv4_pool_bytes(None) == 0


def good():
    """Arguments that pass every check up to the launch; the addresses are never used."""
    cache = b.LLKV4Cache(0x10000, 1 << 40, 2, 64, 16, 8)
    rows = b.LLKV4Rows(None, 0x1000, 0x2000, 3, 1, 3, 8, 0)
    view = b.LLKV4View(0x3000, 4 * 64, 64)
    return cache, rows, view


BAD = [
    ("cache.pool", None, b.LL_E_BAD_ARG), ("cache.pool", 0x10010, b.LL_E_WORKSPACE), ("cache.pool_bytes", 100, b.LL_E_WORKSPACE),
    ("cache.n_kv_heads", 0, b.LL_E_BAD_CONFIG), ("cache.head_dim", 32, b.LL_E_BAD_CONFIG), ("cache.page_tokens", 0, b.LL_E_BAD_CONFIG),
    ("cache.page_tokens", 1 << 30, b.LL_E_BAD_CONFIG), ("cache.n_pages", -1, b.LL_E_BAD_CONFIG),
    ("rows.n_seqs", -1, b.LL_E_BAD_ARG), ("rows.n_rows", -1, b.LL_E_BAD_ARG), ("rows.n_rows", 4, b.LL_E_BAD_ARG),
    ("rows.max_rows", 0, b.LL_E_BAD_ARG), ("rows.table_stride", 0, b.LL_E_BAD_ARG), ("rows.max_len", -1, b.LL_E_BAD_ARG),
    ("rows.len", None, b.LL_E_BAD_ARG), ("rows.page_table", None, b.LL_E_BAD_ARG),
    ("view.data", None, b.LL_E_BAD_ARG), ("view.data", 0x3001, b.LL_E_BAD_ARG), ("view.row_stride", -64, b.LL_E_BAD_ARG),
    ("view.head_stride", -64, b.LL_E_BAD_ARG)]


@pytest.mark.parametrize("what,value,code", BAD)
@pytest.mark.parametrize("call", ["write", "read", "attention"])
def test_bad_arguments_are_refused(call, what, value, code):
    cache, rows, view = good()
    part, field = what.split(".")
    setattr(dict(cache=cache, rows=rows, view=view)[part], field, value)
    c, r, v = C.byref(cache), C.byref(rows), C.byref(view)
    fine = C.byref(b.LLKV4View(0x9000, 256, 64))
    lib = b.load()
    if call == "attention":
        rcs = [lib.ll_kv4_attention(c, r, 0, 4, 0.0, v, None, None, v, None, 0, None)]
        if part == "view":
            rcs += [lib.ll_kv4_attention(c, r, 0, 4, 0.0, fine, *x, None, 0, None) for x in ((None, None, v), (v, fine, fine), (fine, v, fine))]
    else:
        f = getattr(lib, "ll_kv4_" + call)
        rcs = [f(c, r, 0, *x, None) for x in ((v, v), (v, fine), (fine, v)) if part == "view" or x == (v, v)]
    assert set(rcs) == {code} and "ll_kv4_" + call in b.ll_last_error()


def test_other_refusals():
    cache, rows, view = good()
    c, r, v = C.byref(cache), C.byref(rows), C.byref(view)
    lib = b.load()
    att = lib.ll_kv4_attention
    assert lib.ll_kv4_write(None, r, 0, v, v, None) == b.LL_E_BAD_ARG
    assert lib.ll_kv4_write(c, None, 0, v, v, None) == b.LL_E_BAD_ARG
    assert lib.ll_kv4_write(c, r, 2, v, v, None) == b.LL_E_BAD_ARG
    assert lib.ll_kv4_read(c, r, -1, v, v, None) == b.LL_E_BAD_ARG
    assert lib.ll_kv4_write(c, r, 0, None, v, None) == b.LL_E_BAD_ARG
    for heads in (0, 3, -2, 1 << 20):
        assert att(c, r, 0, heads, 0.0, v, None, None, v, None, 0, None) == b.LL_E_BAD_CONFIG
    for scale in (-1.0, float("nan"), float("inf")):
        assert att(c, r, 0, 4, scale, v, None, None, v, None, 0, None) == b.LL_E_BAD_ARG
    assert att(c, r, 0, 4, 0.0, v, v, None, v, None, 0, None) == b.LL_E_BAD_ARG
    assert att(c, r, 0, 4, 0.0, v, None, v, v, None, 0, None) == b.LL_E_BAD_ARG
    # outputs whose elements would overlap; the same strides are fine for an input
    for strides in ((256, 32), (60, 64), (64, 64), (0, 64)):
        bad = C.byref(b.LLKV4View(0x3000, *strides))
        assert att(c, r, 0, 4, 0.0, v, None, None, bad, None, 0, None) == b.LL_E_BAD_ARG, strides
        assert lib.ll_kv4_read(c, r, 0, v, bad, None) == b.LL_E_BAD_ARG, strides
    rows.n_seqs = rows.n_rows = 1 << 24
    assert lib.ll_kv4_write(c, r, 0, v, v, None) == b.LL_E_BAD_ARG


def test_sizes_that_would_leave_32_bits_are_refused():
    cache, rows, view = good()
    c, r, v = C.byref(cache), C.byref(rows), C.byref(view)
    lib = b.load()
    rows.table_stride = (1 << 26) + 1                            # of 16 positions
    assert lib.ll_kv4_attention(c, r, 0, 4, 0.0, v, None, None, v, None, 0, None) == b.LL_E_BAD_ARG and "page table" in b.ll_last_error()
    rows.table_stride, cache.n_kv_heads = 8, 1
    rows.n_seqs, rows.n_rows, rows.max_rows = 1, 1 << 20, 1 << 20
    assert lib.ll_kv4_attention(c, r, 0, 2048, 0.0, v, None, None, v, None, 0, None) == b.LL_E_BAD_ARG and "rows" in b.ll_last_error()
    for field in ("len", "page_table", "row_start"):
        cache, rows, view = good()
        setattr(rows, field, 0x5002)
        assert lib.ll_kv4_write(C.byref(cache), C.byref(rows), 0, C.byref(view), C.byref(view), None) == b.LL_E_BAD_ARG
        assert "aligned" in b.ll_last_error()


def test_nothing_to_do_is_no_error():
    cache, rows, _ = good()
    rows.n_seqs = rows.n_rows = 0
    lib = b.load()
    assert lib.ll_kv4_write(C.byref(cache), C.byref(rows), 0, None, None, None) == b.LL_OK
    assert lib.ll_kv4_read(C.byref(cache), C.byref(rows), 1, None, None, None) == b.LL_OK
    assert lib.ll_kv4_attention(C.byref(cache), C.byref(rows), 0, 4, 0.0, None, None, None, None, None, 0, None) == b.LL_OK


def test_tensors_that_are_not_on_a_gpu_are_refused():
    with pytest.raises(ValueError):
        b.KV4Cache(torch.zeros(1 << 16, dtype=torch.uint8), 2, 64, 16, 2)
    with pytest.raises(ValueError):
        b.KV4Rows(torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32))


def test_definition_holds_what_it_promises():
    """The reference quantiser itself: s has 8 bits and is the smallest that spans the group, values are near."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(500, 128, generator=g).half() * torch.exp2(torch.randint(-20, 12, (500, 1), generator=g).float()).half()
    c, s, mid = ku.quantise(x)
    y = x.double().reshape(500, 4, 32)
    span = y.max(-1).values - y.min(-1).values
    assert (15 * s >= span).all() and (s.half().double() == s).all()
    m, _ = torch.frexp(s)
    assert ((m * 256) == (m * 256).round()).all()
    smaller = torch.nextafter(s.half(), torch.zeros_like(s).half()).double()
    eight = torch.frexp(smaller)[0] * 256
    assert ((15 * smaller < span) | (eight != eight.round()))[s > 0].all()
    off = (ku.values(c, s, mid) - x.double()).abs().reshape(500, 4, 32)
    assert (off <= (s / 2 + mid.abs() * 2.0 ** -11 + 2.0 ** -25)[..., None]).all()


def test_batch_calls_with_a_choice_of_bits_need_an_instance():
    lib = b.load()
    out = (C.c_float * 4)()
    assert lib.ll_batch_pool_bytes_kv(16, 8, 4) == 0
    assert lib.ll_batch_open_kv(4, 16, 8, 4, C.c_void_p(256), 1 << 20) == b.LL_E_NOT_INIT
    assert lib.ll_batch_dbg_get_kv(0, 0, 0, 1, out) == b.LL_E_NOT_INIT
