"""GPU parity of the norm and rotation of queries and keys (bct_norm_rotate and its backward) against the formulas in
64 bits.

Tolerances.  Forward: the mean's sum, the root, two products and the turn are about head_dim/4 + 16 roundings of fp32 on
|x r w| <= sqrt(d) |w|; the sine's argument is a fraction of a turn rounded to fp32, 2 pi 2^-25 of the vector's length.
With m = |y_a| + |y_b| (the pair that is turned) 64 * 2^-24 m covers both; bfloat16 adds half a step, 2^-8 |ref|.
Backward: dx = r (n - xh mean(n xh)); its terms are r |n| and r |xh| mean|n xh|, each with the same count of roundings.
"""
import pytest
import torch

from paper_2411_15785_b200 import binding as B
from paper_2411_15785_b200 import build as bld

import _linear_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _built():
    bld.build()
    B.load()


def _inputs(N, Hq, Hkv, d, dtype, rot, far, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k = (3 * n(N, Hq, d)).to(DT[dtype]), (0.1 * n(N, Hkv, d)).to(DT[dtype])
    wq, wk = (1 + 0.3 * n(d)).to(DT[dtype]), (1 + 0.3 * n(d)).to(DT[dtype])
    pos = torch.randint(0, far, (N,), generator=g, device="cuda")
    freq = 10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) / max(rot // 2, 1)) if rot else None
    return q, k, wq, wk, pos, freq


def _pair_size(y, rot, interleaved):
    """|y_a| + |y_b| for every feature (its own magnitude where it is not turned)."""
    m = y.abs()
    if rot:
        half = rot // 2
        ia = torch.arange(half, device=y.device) * 2 if interleaved else torch.arange(half, device=y.device)
        ib = ia + 1 if interleaved else ia + half
        s = m[..., ia] + m[..., ib]
        m = m.clone()
        m[..., ia], m[..., ib] = s, s
    return m


CASES = [(1, 1, 1, 64, "f32", 64, False), (1, 4, 2, 128, "bf16", 128, False), (7, 3, 1, 128, "f32", 128, True),
         (65, 32, 8, 128, "bf16", 128, False), (33, 5, 5, 64, "bf16", 32, True), (130, 8, 2, 64, "f32", 16, False),
         (501, 7, 1, 128, "bf16", 96, False), (501, 7, 1, 128, "bf16", 48, True), (9, 2, 2, 128, "f32", 0, False),
         (2500, 6, 3, 128, "bf16", 64, False), (2501, 9, 2, 64, "f32", 64, True)]


@pytest.mark.parametrize("N,Hq,Hkv,d,dtype,rot,inter", CASES)
@pytest.mark.parametrize("far", [1, 5000, 1 << 30])
def test_forward_matches_the_formula(N, Hq, Hkv, d, dtype, rot, inter, far):
    q, k, wq, wk, pos, freq = _inputs(N, Hq, Hkv, d, dtype, rot, far, 3 + N)
    out = B.norm_rotate(q, k, wq, wk, pos, freq, eps=1e-5, interleaved=inter)
    for x, w, y in ((q, wq, out[0]), (k, wk, out[1])):
        ref = R.norm_rotate(x, w, pos, freq, 1e-5, inter)
        m = _pair_size(R.norm_rotate(x, w, None, None, 1e-5, inter), rot, inter)
        tol = 64 * 2.0 ** -24 * m + (2.0 ** -8 * ref.abs() if dtype == "bf16" else 0)
        assert y.shape == x.shape and y.dtype == x.dtype
        assert bool(((y.double() - ref).abs() <= tol).all()), float(((y.double() - ref).abs() / tol.clamp(min=1e-30)).max())


def test_no_weights_no_rotation_negative_positions_and_zero_vectors():
    q, k, _, _, pos, freq = _inputs(19, 2, 2, 64, "f32", 64, 100, 5)
    q[3], k[0, 1] = 0, 0
    a = B.norm_rotate(q, k, None, None, None, None, eps=1e-6)
    for x, y in ((q, a[0]), (k, a[1])):
        assert bool(((y.double() - R.norm_rotate(x, None, None, None, 1e-6, False)).abs() <= 1e-5).all())
    assert not bool(a[0][3].any())
    b = B.norm_rotate(q, k, None, None, -pos, freq)
    ref = R.norm_rotate(q, None, -pos, freq, 1e-6, False)
    assert bool(((b[0].double() - ref).abs() <= 128 * 2.0 ** -24 * ref.abs().amax()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_token_dimensions(dtype):
    q, k, wq, wk, pos, freq = _inputs(60, 4, 2, 128, dtype, 128, 999, 9)
    want = B.norm_rotate(q, k, wq, wk, pos, freq)
    q4, k4 = q.view(3, 20, 4, 128).clone(), k.view(3, 20, 2, 128).clone()
    got = B.norm_rotate(q4, k4, wq, wk, pos.view(3, 20), freq, out=(q4, k4))
    assert got[0].data_ptr() == q4.data_ptr()
    assert torch.equal(q4.view_as(q), want[0]) and torch.equal(k4.view_as(k), want[1])


@pytest.mark.parametrize("N,Hq,Hkv,d,dtype,rot,inter", CASES)
def test_backward_matches_the_formula(N, Hq, Hkv, d, dtype, rot, inter):
    q, k, wq, wk, pos, freq = _inputs(N, Hq, Hkv, d, dtype, rot, 5000, 13 + N)
    g = torch.Generator(device="cuda").manual_seed(N)
    dq, dk = (torch.randn(x.shape, generator=g, device="cuda").to(x.dtype) for x in (q, k))
    got = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq, eps=1e-5, interleaved=inter)
    for x, w, dy, dx, dw in ((q, wq, dq, got[0], got[2]), (k, wk, dk, got[1], got[3])):
        lx, lw = x.double().requires_grad_(), w.double().requires_grad_()
        y = R.norm_rotate(lx, lw, pos, freq, 1e-5, inter)
        rx, rw = torch.autograd.grad((y * dy.double()).sum(), (lx, lw))
        xd = x.double()
        r = 1 / torch.sqrt(xd.square().mean(-1, keepdim=True) + 1e-5)
        xh = (xd * r).abs()
        gg = _pair_size(dy.double(), rot, inter)                  # |g| <= |d_a| + |d_b|
        n = gg * w.double().abs()
        mag = r * (n + xh * (n * xh).mean(-1, keepdim=True))
        tol = 96 * 2.0 ** -24 * mag + (2.0 ** -8 * rx.abs() if dtype == "bf16" else 0)
        assert bool(((dx.double() - rx).abs() <= tol).all()), float(((dx.double() - rx).abs() / tol).max())
        # d_w: a lane adds at most N * H terms in fp32, the blocks' shares are added in double
        mw = (gg * xh).sum((0, 1))
        assert bool(((dw.double() - rw).abs() <= (N * x.shape[1] + 64) * 2.0 ** -24 * mw).all())


def test_backward_agrees_with_differences():
    q, k, wq, wk, pos, freq = _inputs(11, 3, 2, 64, "f32", 32, 50, 21)
    k = k * 10
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda x: torch.randn(x.shape, generator=g, device="cuda")
    dq, dk = rnd(q), rnd(k)
    got = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq)

    def loss(a, b, u, w):
        return float((R.norm_rotate(a, u, pos, freq, 1e-6, False) * dq.double()).sum()
                     + (R.norm_rotate(b, w, pos, freq, 1e-6, False) * dk.double()).sum())
    base = [x.double() for x in (q, k, wq, wk)]
    for i in range(4):
        dirn = rnd(base[i]).double()
        h = 1e-5      # the third derivative's share is h^2 ~ 1e-10, the difference's rounding 2^-53 / h ~ 1e-11
        hi, lo = list(base), list(base)
        hi[i], lo[i] = base[i] + h * dirn, base[i] - h * dirn
        num = (loss(*hi) - loss(*lo)) / (2 * h)
        size = float((got[i].double() * dirn).abs().sum())
        assert abs(num - float((got[i].double() * dirn).sum())) <= 128 * 2.0 ** -24 * size + 1e-6 * size, i


def test_backward_in_place_without_weights_gradients_and_repeated():
    q, k, wq, wk, pos, freq = _inputs(700, 4, 2, 128, "bf16", 128, 5000, 31)
    dq, dk = torch.randn_like(q.float()).to(q.dtype), torch.randn_like(k.float()).to(k.dtype)
    a = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq)
    b = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq)
    assert all(torch.equal(x, y) for x, y in zip(a, b))          # the weights' sums have a fixed order
    c = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq, want_d_w=False)
    assert torch.equal(c[0], a[0]) and torch.equal(c[1], a[1]) and c[2] is None
    d = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq, out=(dq, dk, a[2], a[3]))
    assert d[0].data_ptr() == dq.data_ptr() and torch.equal(dq, b[0]) and torch.equal(dk, b[1])
    assert torch.equal(d[2], b[2]) and torch.equal(d[3], b[3])


def test_in_a_replayed_graph_on_another_stream_and_with_bands():
    q, k, wq, wk, pos, freq = _inputs(50, 4, 2, 128, "bf16", 128, 5000, 37)
    s = torch.cuda.Stream()
    want = B.norm_rotate(q, k, wq, wk, pos, freq)
    s.wait_stream(torch.cuda.current_stream())
    got = B.norm_rotate(q, k, wq, wk, pos, freq, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    raw = torch.full((q.numel() * 2 + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    mid = raw[4096:-4096].view(torch.bfloat16).view(q.shape)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.norm_rotate(q, k, wq, wk, pos, freq, out=(mid, torch.empty_like(k)))
    pos.add_(17)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(mid, B.norm_rotate(q, k, wq, wk, pos, freq)[0])
    assert bool((raw[:4096] == 0xA5).all()) and bool((raw[-4096:] == 0xA5).all())


def test_rotated_queries_and_keys_go_into_the_bounded_cache():
    # the other attention step of the library takes them as they are
    Bt, T, Hq, Hkv, d, C = 2, 40, 4, 2, 128, 64
    q, k, wq, wk, _, freq = _inputs(Bt * T, Hq, Hkv, d, "bf16", 128, 10, 41)
    pos = torch.arange(T, device="cuda").repeat(Bt, 1)
    q, k = B.norm_rotate(q.view(Bt, T, Hq, d), k.view(Bt, T, Hkv, d), wq, wk, pos, freq)
    v = torch.randn_like(k.float()).to(k.dtype)
    cache = B.Cache(Bt, Hq, Hkv, d, C, torch.bfloat16)
    out = cache.prefill_stream(q, k, v)
    cache.check_status()
    # C >= T from an empty cache is full causal attention; every output is a mean of at most T values
    qf, kf, vf = (x.double().transpose(1, 2) for x in (q, k, v))
    kf, vf = (x.repeat_interleave(Hq // Hkv, 1) for x in (kf, vf))
    s = (qf @ kf.transpose(-1, -2)) * d ** -0.5
    s = s.masked_fill(~torch.tril(torch.ones(T, T, dtype=torch.bool, device="cuda")), float("-inf"))
    ref = (torch.softmax(s, -1) @ vf).transpose(1, 2)
    assert float((out.double() - ref).abs().max()) <= 2e-2
    cache.destroy()


@pytest.mark.parametrize("N,Hq,Hkv,d,dtype", [(1, 1, 1, 128, "bf16"), (50, 3, 1, 128, "bf16"), (700, 7, 5, 128, "bf16"), (33, 2, 1, 64, "bf16"),
                                              (2500, 7, 3, 64, "bf16"), (90, 3, 1, 64, "f32"), (20, 5, 1, 128, "f32"), (60, 8, 4, 64, "bf16")])
@pytest.mark.parametrize("inter", [False, True])
def test_without_eps_whatever_the_number_of_heads(N, Hq, Hkv, d, dtype, inter):
    # no vector is zero, so nothing is divided by zero; the bounds are those of the tests above
    q, k, wq, wk, pos, freq = _inputs(N, Hq, Hkv, d, dtype, d, 5000, 43 + N)
    g = torch.Generator(device="cuda").manual_seed(N)
    dq, dk = (torch.randn(x.shape, generator=g, device="cuda").to(x.dtype) for x in (q, k))
    out = B.norm_rotate(q, k, wq, wk, pos, freq, eps=0.0, interleaved=inter)
    got = B.norm_rotate_backward(dq, dk, q, k, wq, wk, pos, freq, eps=0.0, interleaved=inter)
    for x, w, dy, y, dx, dw in ((q, wq, dq, out[0], got[0], got[2]), (k, wk, dk, out[1], got[1], got[3])):
        lx, lw = x.double().requires_grad_(), w.double().requires_grad_()
        ref = R.norm_rotate(lx, lw, pos, freq, 0.0, inter)
        rx, rw = torch.autograd.grad((ref * dy.double()).sum(), (lx, lw))
        ref = ref.detach()
        half = 2.0 ** -8 if dtype == "bf16" else 0
        m = _pair_size(R.norm_rotate(x, w, None, None, 0.0, inter), d, inter)
        assert bool(((y.double() - ref).abs() <= 64 * 2.0 ** -24 * m + half * ref.abs()).all())
        r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True))
        xh = (x.double() * r).abs()
        gg = _pair_size(dy.double(), d, inter)
        n = gg * w.double().abs()
        mag = r * (n + xh * (n * xh).mean(-1, keepdim=True))
        assert bool(((dx.double() - rx).abs() <= 96 * 2.0 ** -24 * mag + half * rx.abs()).all())
        mw = (gg * xh).sum((0, 1))
        assert bool(((dw.double() - rw).abs() <= (N * x.shape[1] + 64) * 2.0 ** -24 * mw).all())
