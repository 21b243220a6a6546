"""Refusals of the paged cache operators: every bad argument is turned down before any
device work, so no GPU is needed (the pointers here are never followed)."""
import ctypes

import pytest

import paper_2608_15454_amd as m
from paper_2608_15454_amd import paged

P = 4096  # a stand-in for a device address


@pytest.fixture(scope="module")
def L():
    return m.lib()


def cache(**kw):
    a = dict(dtype=m.F16, n_kv_heads=2, d_head=64, page_size=16, n_pages=4, n_seqs=2, max_pages=3, d_k=P, d_v=P, d_pages=P)
    a.update(kw)
    return paged._Cache(**a)


def rows(**kw):
    a = dict(n_rows=5, max_rows=3, max_slots=40, d_row_start=P, d_first_slot=P)
    a.update(kw)
    return paged._Rows(**a)


def heads(n=2, **kw):
    a = dict(d=P, dtype=m.F32, row_stride=64 * n, head_stride=64)
    a.update(kw)
    return paged._Heads(**a)


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(L, c=None, r=None, n=4, q=None, qo=None, k=None, v=None, pos=None, rope=P, n_pos=99):
    return L.mbp_paged_append(ref(c or cache()), ref(r or rows()), n, ref(q), ref(qo), ref(k or heads()), ref(v or heads()), pos, rope, n_pos, None)


def attend(L, c=None, r=None, n=4, q=None, out=None, lo=None, hi=None, scale=0.125, work=P, size=1 << 30):
    return L.mbp_paged_attend(ref(c or cache()), ref(r or rows()), n, ref(q or heads(4)), ref(out or heads(4)), lo, hi, scale, work, size, None)


BAD_CACHES = [dict(dtype=m.F32), dict(dtype=4), dict(dtype=-1), dict(n_kv_heads=0), dict(n_kv_heads=8193), dict(d_head=48), dict(d_head=256),
              dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(n_pages=0), dict(n_seqs=-1), dict(max_pages=0),
              dict(max_pages=(1 << 26) + 1), dict(d_k=None), dict(d_v=None), dict(d_k=P + 8), dict(d_v=P + 4), dict(d_pages=None), dict(d_pages=P + 2)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches(L, bad):
    c = cache(**bad)
    assert append(L, c) == m.EINVAL and L.mbp_paged_error()
    assert attend(L, c) == m.EINVAL
    assert L.mbp_paged_read(ref(c), ref(rows()), ref(heads()), ref(heads()), None) == m.EINVAL
    if not any(key.startswith("d_") and key != "d_head" for key in bad):
        assert L.mbp_paged_pool_bytes(ref(c)) == 0
        assert L.mbp_paged_workspace_bytes(ref(c), ref(rows()), 4) == 0


@pytest.mark.parametrize("bad", [dict(n_rows=-1), dict(max_rows=-1), dict(max_slots=-1), dict(d_row_start=None), dict(d_first_slot=None),
                                 dict(d_row_start=P + 1), dict(d_first_slot=P + 2)], ids=str)
def test_bad_rows(L, bad):
    r = rows(**bad)
    assert append(L, r=r) == m.EINVAL and attend(L, r=r) == m.EINVAL
    assert L.mbp_paged_read(ref(cache()), ref(r), ref(heads()), ref(heads()), None) == m.EINVAL


@pytest.mark.parametrize("bad", [dict(d=None), dict(dtype=m.MXFP4), dict(dtype=9), dict(d=P + 2), dict(row_stride=-1), dict(head_stride=-64),
                                 dict(row_stride=1 << 41)], ids=str)
def test_bad_heads(L, bad):
    assert append(L, k=heads(**bad)) == m.EINVAL and append(L, v=heads(**bad)) == m.EINVAL
    assert append(L, q=heads(4, **bad), qo=heads(4)) == m.EINVAL and append(L, q=heads(4), qo=heads(4, **bad)) == m.EINVAL
    assert attend(L, q=heads(4, **bad)) == m.EINVAL and attend(L, out=heads(4, **bad)) == m.EINVAL
    assert L.mbp_paged_read(ref(cache()), ref(rows()), ref(heads(**bad)), ref(heads()), None) == m.EINVAL


@pytest.mark.parametrize("rs,hs", [(0, 64), (256, 0), (256, 63), (255, 64), (64, 64), (64, 256), (63, 64 * 5)])
def test_outputs_whose_heads_overlap(L, rs, hs):
    """5 rows of 4 heads of 64 channels."""
    o = heads(4, row_stride=rs, head_stride=hs)
    assert attend(L, out=o) == m.EINVAL and b"overlap" in L.mbp_paged_error()
    assert append(L, q=heads(4), qo=o) == m.EINVAL
    two = heads(2, row_stride=min(rs, 127), head_stride=hs)
    assert L.mbp_paged_read(ref(cache()), ref(rows()), ref(two), ref(heads()), None) == m.EINVAL


def test_heads_and_types_that_do_not_go_together(L):
    assert attend(L, n=3) == m.EINVAL and attend(L, n=0) == m.EINVAL and attend(L, n=8194) == m.EINVAL
    assert attend(L, q=heads(4, dtype=m.F16)) == m.EINVAL  # out is float32
    assert attend(L, q=heads(4, dtype=m.BF16), out=heads(4, dtype=m.BF16)) == m.EINVAL  # over a float16 cache
    assert append(L, q=heads(4)) == m.EINVAL and append(L, qo=heads(4)) == m.EINVAL
    assert append(L, n=3, q=heads(3), qo=heads(3)) == m.EINVAL
    assert append(L, q=heads(4), qo=heads(4, dtype=m.F16)) == m.EINVAL
    assert append(L, q=heads(4), qo=heads(4, row_stride=512)) == m.EINVAL  # q itself, with other strides


def test_bad_tables_ranges_and_scales(L):
    assert append(L, rope=P + 8) == m.EINVAL and append(L, n_pos=0) == m.EINVAL
    assert append(L, pos=P, rope=None) == m.EINVAL and append(L, pos=P + 2) == m.EINVAL
    assert attend(L, lo=P + 1) == m.EINVAL and attend(L, hi=P + 3) == m.EINVAL
    assert attend(L, scale=float("nan")) == m.EINVAL and attend(L, scale=float("inf")) == m.EINVAL
    for bad in ((None, 9, 64, 1e5), (P + 4, 9, 64, 1e5), (P, 0, 64, 1e5), (P, 9, 48, 1e5), (P, 9, 64, 0.0), (P, 9, 64, float("inf"))):
        assert L.mbp_rope_table(*bad, None) == m.EINVAL


def test_workspaces(L):
    c, r = cache(n_pages=4096, max_pages=2048), rows(n_rows=2, max_rows=1, max_slots=32768)
    need = L.mbp_paged_workspace_bytes(ref(c), ref(r), 4)
    assert need > 0 and need % ((64 + 2) * 4 * 2 * 4) == 0  # a whole number of splits
    assert attend(L, c, r, work=None) == m.EINVAL and attend(L, c, r, work=P + 8) == m.EINVAL
    assert attend(L, c, r, size=need - 1) == m.ECAPACITY
    assert L.mbp_paged_workspace_bytes(ref(c), ref(rows(max_slots=16)), 4) == 0
    # bounds beyond the cache's and the call's rows ask for no more than those
    assert L.mbp_paged_workspace_bytes(ref(c), ref(rows(n_rows=2, max_rows=2, max_slots=2**31 - 1)), 4) == \
        L.mbp_paged_workspace_bytes(ref(c), ref(rows(n_rows=2, max_rows=2**31 - 1, max_slots=32768)), 4)


def test_nothing_to_do_is_no_error(L):
    assert append(L, r=rows(n_rows=0)) == m.OK and attend(L, r=rows(n_rows=0)) == m.OK
    empty = cache(n_seqs=0, d_pages=None)
    assert append(L, empty, rows(d_row_start=None, d_first_slot=None)) == m.OK
    assert attend(L, empty, rows(d_row_start=None, d_first_slot=None)) == m.OK
    assert attend(L, r=rows(max_rows=0)) == m.OK
    assert L.mbp_paged_read(ref(cache()), ref(rows(n_rows=0)), ref(heads()), ref(heads()), None) == m.OK


def test_calls_too_large_for_a_launch(L):
    big = rows(n_rows=2**31 - 1, max_rows=2**31 - 1)
    wide = heads(8192, row_stride=8192 * 64)
    c = cache(n_kv_heads=8192)
    assert append(L, c, big, k=wide, v=wide) == m.ECAPACITY
    assert attend(L, c, big, n=8192, q=wide, out=wide) == m.ECAPACITY


def test_pool_bytes(L):
    for dtype, slot in ((m.F16, 128), (m.BF16, 128), (m.MXFP4, 34)):
        assert L.mbp_paged_pool_bytes(ref(cache(dtype=dtype))) == 4 * 2 * 16 * slot


def test_scales_beyond_float32_in_base_two(L):
    assert attend(L, scale=2.5e38) == m.EINVAL and attend(L, scale=-2.5e38) == m.EINVAL


def test_out_in_the_place_of_q(L):
    assert attend(L, q=heads(4), out=heads(4, row_stride=999)) == m.EINVAL
    assert b"place of q" in L.mbp_paged_error()
