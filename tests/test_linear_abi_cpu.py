"""Host-side checks of the linear-attention and norm/rotation calls: sizes, refusals, all before a device is touched."""
import ctypes
import gc
import weakref

import pytest
import torch

from paper_2411_15785_b200 import binding as B
from paper_2411_15785_b200 import build as bld


@pytest.fixture(scope="module")
def lib():
    bld.build()
    return B.load()


def _p(batch=2, Hq=4, Hkv=2, d=128, dtype=B.BCT_BF16, scale=0.0):
    return B.BctLinearParams(batch, Hq, Hkv, d, dtype, scale)


# addresses far enough apart that nothing overlaps; none is dereferenced by a refused call
A = [(i + 1) << 34 for i in range(16)]


def _step(lib, p, **kw):
    a = dict(q=A[0], k=A[1], v=A[2], decay=A[3], state=A[4], state_out=A[4], out=A[5])
    a.update(kw)
    return lib.bct_linear_step(ctypes.byref(p) if p is not None else None, a["q"], a["k"], a["v"], a["decay"], a["state"],
                               a["state_out"], a["out"], None)


def _fwd(lib, p, T=8, **kw):
    a = dict(q=A[0], k=A[1], v=A[2], decay=A[3], lens=None, state=A[4], state_out=A[5], out=A[6], scratch=A[7], n=1 << 33)
    a.update(kw)
    return lib.bct_linear_forward(ctypes.byref(p), T, a["q"], a["k"], a["v"], a["decay"], a["lens"], a["state"],
                                  a["state_out"], a["out"], a["scratch"], a["n"], None)


def _bwd(lib, p, T=8, **kw):
    a = dict(d_out=A[0], q=A[1], k=A[2], v=A[3], decay=A[4], lens=None, state=A[5], d_state=A[6], d_q=A[7], d_k=A[8],
             d_v=A[9], d_in=A[10], scratch=A[11], n=1 << 33)
    a.update(kw)
    return lib.bct_linear_backward(ctypes.byref(p), T, *[a[x] for x in ("d_out", "q", "k", "v", "decay", "lens", "state",
                                                                          "d_state", "d_q", "d_k", "d_v", "d_in", "scratch",
                                                                          "n")], None)


def test_params_struct_matches_header_layout():
    assert ctypes.sizeof(B.BctLinearParams) == 6 * 4


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), B.BCT_ERR_INVALID_ARG),
    (dict(Hq=5), B.BCT_ERR_INVALID_ARG),
    (dict(Hkv=0), B.BCT_ERR_INVALID_ARG),
    (dict(dtype=7), B.BCT_ERR_INVALID_ARG),
    (dict(dtype=B.BCT_BF16_PAIR), B.BCT_ERR_INVALID_ARG),
    (dict(d=96), B.BCT_ERR_UNSUPPORTED),
    (dict(scale=float("inf")), B.BCT_ERR_INVALID_ARG),
    (dict(scale=1e-45), B.BCT_ERR_INVALID_ARG),        # its reciprocal is not finite
    (dict(batch=1 << 20, Hkv=2, Hq=2), B.BCT_ERR_INVALID_ARG),
])
def test_bad_linear_params_are_refused_by_every_call(lib, kw, status):
    p = _p(**kw)
    n = ctypes.c_size_t(0)
    assert lib.bct_linear_scratch_bytes(ctypes.byref(p), 8, 0, ctypes.byref(n)) == status
    assert _step(lib, p) == status and _fwd(lib, p) == status and _bwd(lib, p) == status
    assert B.last_error() != ""


def test_null_and_misaligned_operands_are_refused(lib):
    p = _p()
    assert _step(lib, None) == B.BCT_ERR_INVALID_ARG
    for name in ("q", "k", "v", "decay", "state", "state_out", "out"):
        assert _step(lib, p, **{name: None}) == B.BCT_ERR_INVALID_ARG, name
        assert _step(lib, p, **{name: A[9] + 2}) == B.BCT_ERR_INVALID_ARG, name
    for name in ("q", "k", "v", "decay", "out"):
        assert _fwd(lib, p, **{name: None}) == B.BCT_ERR_INVALID_ARG, name
    for name in ("q", "k", "v", "state", "state_out", "out"):
        assert _fwd(lib, p, **{name: A[9] + 8}) == B.BCT_ERR_INVALID_ARG, name
    assert _fwd(lib, p, lens=A[9] + 2) == B.BCT_ERR_INVALID_ARG
    for name in ("d_out", "q", "k", "v", "decay", "d_q", "d_k", "d_v"):
        assert _bwd(lib, p, **{name: None}) == B.BCT_ERR_INVALID_ARG, name
    for T in (0, -1, (1 << 30) + 1):
        assert _fwd(lib, p, T=T) == B.BCT_ERR_INVALID_ARG and _bwd(lib, p, T=T) == B.BCT_ERR_INVALID_ARG


def test_overlapping_operands_are_refused(lib):
    p = _p()
    kv, q, st = 2 * 2 * 128 * 2, 2 * 4 * 128 * 2, 2 * 2 * 128 * 128 * 4
    assert _step(lib, p, out=A[0]) == B.BCT_ERR_INVALID_ARG and "overlaps" in B.last_error()
    assert _step(lib, p, out=A[1] + kv - 16) == B.BCT_ERR_INVALID_ARG
    assert _step(lib, p, state_out=A[4] + 16) == B.BCT_ERR_INVALID_ARG      # in place means exactly in place
    assert _step(lib, p, out=A[4] + st - 16) == B.BCT_ERR_INVALID_ARG
    assert _fwd(lib, p, out=A[0]) == B.BCT_ERR_INVALID_ARG
    assert _fwd(lib, p, out=A[5]) == B.BCT_ERR_INVALID_ARG
    assert _fwd(lib, p, state_out=A[4] + 256) == B.BCT_ERR_INVALID_ARG
    assert _bwd(lib, p, d_in=A[6]) == B.BCT_ERR_INVALID_ARG                 # d_state is still read while d_state_in is written
    assert _bwd(lib, p, d_q=A[0]) == B.BCT_ERR_INVALID_ARG
    assert _bwd(lib, p, d_k=A[9]) == B.BCT_ERR_INVALID_ARG
    assert q  # (sizes above are those of the calls)


def test_scratch_is_sized_checked_and_refused_when_short(lib):
    n = ctypes.c_size_t(0)
    many = _p(batch=64, Hq=32, Hkv=32)
    assert lib.bct_linear_scratch_bytes(ctypes.byref(many), 128, 0, ctypes.byref(n)) == B.BCT_OK and n.value == 0
    few = _p(batch=1, Hq=8, Hkv=2)
    assert lib.bct_linear_scratch_bytes(ctypes.byref(few), 16384, 0, ctypes.byref(n)) == B.BCT_OK
    fwd = n.value
    state = 2 * 128 * 128 * 4
    assert fwd % 256 == 0 and fwd >= 2 * state and fwd <= 64 * state
    assert lib.bct_linear_scratch_bytes(ctypes.byref(few), 16384, 1, ctypes.byref(n)) == B.BCT_OK and n.value >= 2 * state
    assert _fwd(lib, few, T=16384, n=fwd - 1) == B.BCT_ERR_INVALID_ARG and "scratch" in B.last_error()
    assert _fwd(lib, few, T=16384, scratch=None) == B.BCT_ERR_INVALID_ARG
    assert _fwd(lib, few, T=16384, scratch=A[7] + 128) == B.BCT_ERR_INVALID_ARG
    assert _fwd(lib, few, T=16384, scratch=A[0]) == B.BCT_ERR_INVALID_ARG      # on top of q
    assert lib.bct_linear_scratch_bytes(ctypes.byref(few), 16384, 0, None) == B.BCT_ERR_INVALID_ARG
    assert B.linear_scratch_bytes(1, 16384, 8, 2, 128, torch.bfloat16) == fwd


def _nr(lib, n=8, Hq=4, Hkv=2, d=128, dtype=B.BCT_BF16, q=A[0], k=A[1], w_q=A[2], w_k=A[3], eps=1e-6, pos=A[4], freq=A[5],
        rot=128, flags=0, q_out=A[6], k_out=A[7]):
    return lib.bct_norm_rotate(n, Hq, Hkv, d, dtype, q, k, w_q, w_k, eps, pos, freq, rot, flags, q_out, k_out, None)


def _nrb(lib, n=8, Hq=4, Hkv=2, d=128, dtype=B.BCT_BF16, dqo=A[8], dko=A[9], q=A[0], k=A[1], w_q=A[2], w_k=A[3], eps=1e-6,
         pos=A[4], freq=A[5], rot=128, flags=0, d_q=A[6], d_k=A[7], d_w_q=A[10], d_w_k=A[11], scratch=A[12], nb=1 << 30):
    return lib.bct_norm_rotate_backward(n, Hq, Hkv, d, dtype, dqo, dko, q, k, w_q, w_k, eps, pos, freq, rot, flags, d_q, d_k,
                                        d_w_q, d_w_k, scratch, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), B.BCT_ERR_INVALID_ARG), (dict(n=(1 << 30) + 1), B.BCT_ERR_INVALID_ARG),
    (dict(Hq=0), B.BCT_ERR_INVALID_ARG), (dict(Hkv=0), B.BCT_ERR_INVALID_ARG),
    (dict(dtype=2), B.BCT_ERR_INVALID_ARG), (dict(d=96), B.BCT_ERR_UNSUPPORTED),
    (dict(eps=-1.0), B.BCT_ERR_INVALID_ARG), (dict(eps=float("nan")), B.BCT_ERR_INVALID_ARG),
    (dict(rot=-16), B.BCT_ERR_INVALID_ARG), (dict(rot=144), B.BCT_ERR_INVALID_ARG), (dict(rot=40), B.BCT_ERR_UNSUPPORTED),
    (dict(flags=2), B.BCT_ERR_INVALID_ARG), (dict(pos=None), B.BCT_ERR_INVALID_ARG), (dict(freq=None), B.BCT_ERR_INVALID_ARG),
    (dict(pos=A[4] + 4), B.BCT_ERR_INVALID_ARG), (dict(q=None), B.BCT_ERR_INVALID_ARG), (dict(k=A[1] + 8), B.BCT_ERR_INVALID_ARG),
    (dict(w_q=A[2] + 2), B.BCT_ERR_INVALID_ARG),
])
def test_bad_norm_rotate_arguments_are_refused(lib, kw, status):
    assert _nr(lib, **kw) == status
    assert _nrb(lib, **kw) == status


def test_norm_rotate_overlaps_and_scratch(lib):
    assert _nr(lib, q_out=A[0] + 16) == B.BCT_ERR_INVALID_ARG and "overlaps" in B.last_error()
    assert _nr(lib, q_out=A[1]) == B.BCT_ERR_INVALID_ARG       # q's result over k
    assert _nr(lib, k_out=A[6]) == B.BCT_ERR_INVALID_ARG       # both results in one place
    assert _nrb(lib, d_q=A[0]) == B.BCT_ERR_INVALID_ARG
    assert _nrb(lib, nb=16) == B.BCT_ERR_INVALID_ARG and "scratch" in B.last_error()
    assert _nrb(lib, scratch=None) == B.BCT_ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    assert lib.bct_norm_rotate_scratch_bytes(8, 128, ctypes.byref(n)) == B.BCT_OK and n.value >= 2 * 128 * 4
    assert lib.bct_norm_rotate_scratch_bytes(0, 128, ctypes.byref(n)) == B.BCT_ERR_INVALID_ARG
    assert lib.bct_norm_rotate_scratch_bytes(8, 128, None) == B.BCT_ERR_INVALID_ARG


def test_the_binding_refuses_tensors_the_library_cannot_see_the_layout_of():
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64)
    g, s = torch.zeros(2), torch.zeros(2, 2, 64, 64)
    with pytest.raises(ValueError):      # not on a device
        B.linear_step(q, k, k, g, s)
    with pytest.raises(ValueError):
        B.norm_rotate(q, k, None, None, None, None)
    with pytest.raises(ValueError):
        B.linear_step(q.half(), k.half(), k.half(), g, s)


def test_results_over_decays_lengths_positions_or_frequencies_are_refused(lib):
    p = _p()
    assert _step(lib, p, out=A[3] - 16) == B.BCT_ERR_INVALID_ARG and "log_decay" in B.last_error()
    assert _fwd(lib, p, state_out=A[3] - 256) == B.BCT_ERR_INVALID_ARG and "log_decay" in B.last_error()
    assert _fwd(lib, p, lens=A[6] + 16) == B.BCT_ERR_INVALID_ARG and "lens" in B.last_error()
    assert _bwd(lib, p, lens=A[9] + 4) == B.BCT_ERR_INVALID_ARG and "lens" in B.last_error()
    assert _bwd(lib, p, d_k=A[4] - 64) == B.BCT_ERR_INVALID_ARG and "log_decay" in B.last_error()
    assert _nr(lib, k_out=A[4] + 48) == B.BCT_ERR_INVALID_ARG and "positions" in B.last_error()
    assert _nrb(lib, d_q=A[5] + 496) == B.BCT_ERR_INVALID_ARG and "freq" in B.last_error()


def test_a_scale_that_is_not_a_number_is_refused(lib):
    p = _p(scale=float("nan"))
    assert _step(lib, p) == B.BCT_ERR_INVALID_ARG and "scale" in B.last_error()
    assert _fwd(lib, p) == B.BCT_ERR_INVALID_ARG and _bwd(lib, p) == B.BCT_ERR_INVALID_ARG


def test_a_scale_is_read_at_every_call_and_not_kept():
    # (the call is refused, the tensors being on the CPU, but only after its sizes and its scale have been looked at)
    q, k, g, s = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64), torch.zeros(2), torch.zeros(2, 2, 64, 64)
    scale = torch.tensor(0.5)
    kept = weakref.ref(scale)
    with pytest.raises(ValueError):
        B.linear_step(q, k, k, g, s, scale=scale)
    scale.mul_(2)
    sizes = [_scale_of(q, k, x) for x in (scale, 1.0, 0.5)]
    assert sizes == [1.0, 1.0, 0.5]
    del scale
    gc.collect()
    assert kept() is None
    n = torch.tensor(2)
    a = B.linear_scratch_bytes(n, 16384, 8, 2, 128, torch.bfloat16)
    n.fill_(1)
    assert B.linear_scratch_bytes(n, 16384, 8, 2, 128, torch.bfloat16) == B.linear_scratch_bytes(1, 16384, 8, 2, 128, torch.bfloat16)
    assert a == B.linear_scratch_bytes(2, 16384, 8, 2, 128, torch.bfloat16)


def _scale_of(q, k, scale):
    """The scale that a call with these arguments hands to the library."""
    seen = []
    with pytest.MonkeyPatch.context() as m:
        m.setattr(B, "_operand", lambda *a: None)
        m.setattr(B, "_launch", lambda dev, call, p, *a: seen.append(p._obj.scale))
        B.linear_step(q, k, k, torch.zeros(2), torch.zeros(2, 2, 64, 64), scale=scale)
    return seen[0]


def test_a_backward_without_the_state_gradient_needs_no_room_for_it(lib):
    p = _p(batch=8, Hq=32, Hkv=8)
    n = ctypes.c_size_t(0)
    need = []
    for kind in (1, 2):
        assert lib.bct_linear_scratch_bytes(ctypes.byref(p), 4096, kind, ctypes.byref(n)) == B.BCT_OK
        need.append(n.value)
    # every query head's share of d_state_in; the launch of d_q, before it, uses the same place for less
    assert need[0] >= 8 * 32 * 128 * 128 * 4 > need[1]
    bf, f32 = torch.bfloat16, torch.float32
    assert B.linear_scratch_bytes(8, 4096, 32, 8, 128, bf, backward=True) == need[0]
    assert B.linear_scratch_bytes(8, 4096, 32, 8, 128, bf, backward=True, want_d_state=False) == need[1]
    for Hq, dt in ((8, bf), (32, f32)):                    # elsewhere it is no room of its own
        assert B.linear_scratch_bytes(1, 16384, Hq, 8, 128, dt, backward=True) == \
            B.linear_scratch_bytes(1, 16384, Hq, 8, 128, dt, backward=True, want_d_state=False)
    # no more is asked for than that (the refused overlap says that the scratch was taken), and no less
    assert _bwd(lib, p, T=4096, d_in=None, n=need[1], d_q=A[0]) == B.BCT_ERR_INVALID_ARG and "overlaps" in B.last_error()
    assert _bwd(lib, p, T=4096, n=need[1]) == B.BCT_ERR_INVALID_ARG and "scratch" in B.last_error()
    few = _p(batch=1, Hq=32, Hkv=8)
    assert lib.bct_linear_scratch_bytes(ctypes.byref(few), 16384, 2, ctypes.byref(n)) == B.BCT_OK and n.value > 0
    assert _bwd(lib, few, T=16384, d_in=None, n=n.value - 1) == B.BCT_ERR_INVALID_ARG and "scratch" in B.last_error()
