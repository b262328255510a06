"""Host-side checks of the calls of the 8-bit cache: sizes, refusals, all before a device is touched."""
import ctypes

import pytest

from paper_2411_15785_b200 import binding as B
from paper_2411_15785_b200 import build as bld


@pytest.fixture(scope="module")
def lib():
    bld.build()
    return B.load()


# addresses far enough apart that nothing overlaps; none is dereferenced by a refused call
A = [(i + 1) << 36 for i in range(16)]
PLANES = ("k", "v", "k_scale", "v_scale", "weight", "position", "state")


def _c(batch=2, Hkv=2, d=128, C=100, **kw):
    at = dict(zip(PLANES, A))
    at.update(kw)
    return B.BctQcache(batch, Hkv, d, C, *(at[n] for n in PLANES))


def _append(lib, c, T=8, dtype=B.BCT_BF16, k=A[7], v=A[8], lens=None):
    return lib.bct_qcache_append(None if c is None else ctypes.byref(c), T, dtype, k, v, lens, None)


def _attend(lib, c, T=8, Hq=4, dtype=B.BCT_BF16, q=A[7], lens=None, scale=0.0, cap=0.0, acc=1, out=A[8], scratch=A[9], n=1 << 35):
    return lib.bct_qcache_attend(None if c is None else ctypes.byref(c), T, Hq, dtype, q, lens, scale, cap, acc, out, scratch, n,
                                 None)


def _evict(lib, c, keep=50, recent=0, scratch=A[9], n=1 << 35):
    return lib.bct_qcache_evict(None if c is None else ctypes.byref(c), keep, recent, scratch, n, None)


def test_struct_matches_header_layout():
    assert ctypes.sizeof(B.BctQcache) == 4 * 4 + 7 * 8
    assert B.QCACHE_BLOCK == 32


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), B.BCT_ERR_INVALID_ARG), (dict(Hkv=0), B.BCT_ERR_INVALID_ARG), (dict(C=0), B.BCT_ERR_INVALID_ARG),
    (dict(C=(1 << 24) + 1), B.BCT_ERR_INVALID_ARG), (dict(batch=1 << 20), B.BCT_ERR_INVALID_ARG),
    (dict(d=0), B.BCT_ERR_INVALID_ARG), (dict(d=96), B.BCT_ERR_UNSUPPORTED),
])
def test_bad_sizes_are_refused_by_every_call(lib, kw, status):
    c, n = _c(**kw), ctypes.c_size_t(0)
    assert _append(lib, c) == status and _attend(lib, c, Hq=kw.get("Hkv", 2) or 2) == status and _evict(lib, c, keep=0) == status
    assert lib.bct_qcache_attend_scratch_bytes(ctypes.byref(c), 8, 4, B.BCT_BF16, 1, ctypes.byref(n)) == status
    assert lib.bct_qcache_evict_scratch_bytes(ctypes.byref(c), 0, ctypes.byref(n)) == status
    assert B.last_error() != ""


def test_null_and_misaligned_operands_are_refused(lib):
    assert _append(lib, None) == _attend(lib, None) == _evict(lib, None) == B.BCT_ERR_INVALID_ARG
    for name in PLANES:
        for bad in (None, A[10] + 8):
            c = _c(**{name: bad})
            assert _append(lib, c) == _attend(lib, c) == _evict(lib, c) == B.BCT_ERR_INVALID_ARG, name
            assert name in B.last_error()
    c = _c()
    for bad in (None, A[10] + 8):
        assert _append(lib, c, k=bad) == _append(lib, c, v=bad) == B.BCT_ERR_INVALID_ARG
        assert _attend(lib, c, q=bad) == _attend(lib, c, out=bad) == B.BCT_ERR_INVALID_ARG
    assert _append(lib, c, lens=A[10] + 2) == _attend(lib, c, lens=A[10] + 2) == B.BCT_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(T=0), dict(T=-1), dict(T=1 << 31), dict(dtype=2), dict(dtype=7)])
def test_bad_token_counts_and_types_are_refused(lib, kw):
    n = ctypes.c_size_t(0)
    assert _append(lib, _c(), **kw) == _attend(lib, _c(), **kw) == B.BCT_ERR_INVALID_ARG
    assert lib.bct_qcache_attend_scratch_bytes(ctypes.byref(_c()), kw.get("T", 8), 4, kw.get("dtype", 1), 1,
                                               ctypes.byref(n)) == B.BCT_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(Hq=0), dict(Hq=3), dict(Hq=(1 << 16) + 2), dict(scale=float("nan")), dict(scale=float("inf")),
                                dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e30, scale=1e-30),
                                dict(cap=1e-30, scale=1e30)])
def test_bad_attention_arguments_are_refused(lib, kw):
    assert _attend(lib, _c(), **kw) == B.BCT_ERR_INVALID_ARG


@pytest.mark.parametrize("keep,recent", [(-1, 0), (101, 0), (50, -1), (50, 51), (0, 1)])
def test_bad_eviction_arguments_are_refused(lib, keep, recent):
    assert _evict(lib, _c(), keep=keep, recent=recent) == B.BCT_ERR_INVALID_ARG


def test_overlapping_operands_are_refused(lib):
    plane = 2 * 2 * 100 * 128
    c = _c()
    assert _append(lib, _c(v=A[0] + plane - 16)) == B.BCT_ERR_INVALID_ARG and "overlaps" in B.last_error()
    assert _append(lib, c, k=A[0] + 16) == B.BCT_ERR_INVALID_ARG
    assert _append(lib, c, lens=A[6]) == B.BCT_ERR_INVALID_ARG
    assert _attend(lib, c, out=A[7]) == B.BCT_ERR_INVALID_ARG         # not in place: rows share their keys' warps
    assert _attend(lib, c, out=A[4]) == B.BCT_ERR_INVALID_ARG
    assert _attend(lib, c, scratch=A[8]) == B.BCT_ERR_INVALID_ARG
    assert _attend(lib, c, scratch=A[1]) == B.BCT_ERR_INVALID_ARG
    assert _evict(lib, c, scratch=A[4]) == B.BCT_ERR_INVALID_ARG
    assert _evict(lib, _c(weight=A[5])) == B.BCT_ERR_INVALID_ARG


def test_scratch_is_sized_checked_and_refused_when_short(lib):
    n = ctypes.c_size_t(0)
    c = _c(batch=3, Hkv=4, C=5000)
    for T, acc in ((1, 0), (1, 1), (700, 1)):
        assert lib.bct_qcache_attend_scratch_bytes(ctypes.byref(c), T, 8, B.BCT_BF16, acc, ctypes.byref(n)) == B.BCT_OK
        assert n.value > 0 and n.value % 256 == 0
        assert _attend(lib, c, T=T, Hq=8, acc=acc, n=n.value - 1) == B.BCT_ERR_INVALID_ARG and "scratch" in B.last_error()
        assert _attend(lib, c, T=T, Hq=8, acc=acc, scratch=None) == B.BCT_ERR_INVALID_ARG
        assert _attend(lib, c, T=T, Hq=8, acc=acc, scratch=A[9] + 128) == B.BCT_ERR_INVALID_ARG
    assert lib.bct_qcache_evict_scratch_bytes(ctypes.byref(c), 4000, ctypes.byref(n)) == B.BCT_OK
    assert 12 * 1000 * 4 <= n.value <= 12 * 1000 * 24 + 8192
    assert _evict(lib, c, keep=4000, n=n.value - 1) == B.BCT_ERR_INVALID_ARG
    assert _evict(lib, c, keep=4000, scratch=None) == B.BCT_ERR_INVALID_ARG
    assert lib.bct_qcache_evict_scratch_bytes(ctypes.byref(c), 5000, ctypes.byref(n)) == B.BCT_OK and n.value == 0
    assert _evict(lib, c, keep=5000, scratch=None, n=0) == B.BCT_OK       # no cache holds more: nothing to do
    assert lib.bct_qcache_evict_scratch_bytes(ctypes.byref(c), 5000, None) == B.BCT_ERR_INVALID_ARG
    assert lib.bct_qcache_attend_scratch_bytes(ctypes.byref(c), 1, 8, B.BCT_BF16, 1, None) == B.BCT_ERR_INVALID_ARG
