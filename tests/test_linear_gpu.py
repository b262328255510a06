"""GPU parity of linear attention with a decay for each head (bct_linear_step / _forward / _backward) against the token
loop in 64 bits.

Tolerances.  Let M be the same formula on the absolute values of its inputs: the sum of the magnitudes of every term
that an element adds up.  In fp32 a term goes through at most n roundings (the products and sums over head_dim, over a
chunk, over the chunks before it, the powers of the decay), so the error is at most n 2^-24 M; n is taken as head_dim +
T + 64.  bfloat16: the output is rounded once, 2^-8 |ref|; on the tensor path the products of pairs, and the state where
it enters a product, are rounded to bfloat16 as well, 2^-8 M.  Those roundings are independent, each spread evenly over
its half step (rms 2^-8/sqrt(3) at most): two of them in a row give an rms error of at most sqrt(2/3) 2^-8 = 0.0032 of
the rms of the result where no cancellation is planted, and 0.005 is asked for.
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


def _inputs(Bt, T, Hq, Hkv, d, dtype, seed, decay="spread", state=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[dtype])
    q, k, v = n(Bt, T, Hq, d), n(Bt, T, Hkv, d), n(Bt, T, Hkv, d)
    if decay == "spread":
        ld = -(2.0 ** (-8.0 * torch.arange(1, Hkv + 1, device="cuda") / Hkv)).float()
    else:
        ld = torch.full((Hkv,), float(decay), device="cuda")
    S = torch.randn((Bt, Hkv, d, d), generator=g, device="cuda") if state else None
    return q, k, v, ld, S


def _check(name, got, ref, mag, dtype, n, tensor=False):
    got = got.double()
    assert torch.isfinite(got).all(), name
    tol = n * 2.0 ** -24 * mag + 1e-30
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * ref.abs() + (2.0 ** -8 * mag if tensor else 0.0)
    bad = (got - ref).abs() > tol
    assert not bool(bad.any()), (name, int(bad.sum()), float((got - ref).abs().max()), float(((got - ref).abs() / tol).max()))
    rms = float(ref.square().mean().sqrt())
    if dtype == "bf16" and rms > 0 and ref.numel() >= 4096:
        assert float((got - ref).square().mean().sqrt()) <= 0.005 * rms, name


def _forward_case(Bt, T, Hq, Hkv, d, dtype, seed, decay="spread", lens=None, state=True, scale=0.0):
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, dtype, seed, decay, state)
    lt = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if lens is not None:       # padding holds whatever memory held
        for b, n in enumerate(lens):
            for x in (q, k, v):
                x[b, max(n, 0):] = float("nan")
    out, S1 = B.linear_forward(q, k, v, ld, state=S, lens=lt, scale=scale)
    torch.cuda.synchronize()
    rs = None if scale == 0.0 else scale
    zero = lambda x: torch.nan_to_num(x)
    ref, rS = R.linear_forward(zero(q), zero(k), zero(v), ld, S, lens, rs)
    mag, mS = R.linear_forward(zero(q).abs(), zero(k).abs(), zero(v).abs(), ld, None if S is None else S.abs(), lens, rs)
    n = d + T + 64
    _check("out", out, ref, mag, dtype, n, tensor=True)
    _check("state", S1, rS, mS, "f32", n)
    return q, k, v, ld, S, out, S1


CASES = [
    (1, 1, 1, 1, 64, "f32"), (2, 1, 4, 2, 128, "bf16"), (1, 2, 2, 1, 128, "f32"), (3, 31, 4, 4, 64, "bf16"),
    (2, 32, 2, 2, 128, "f32"), (2, 33, 6, 2, 64, "f32"), (1, 127, 2, 2, 128, "bf16"), (2, 128, 4, 4, 128, "bf16"),
    (2, 129, 8, 2, 128, "bf16"), (1, 300, 7, 1, 128, "bf16"), (1, 333, 15, 1, 64, "bf16"), (1, 511, 2, 1, 128, "f32"),
    (1, 1025, 3, 3, 128, "bf16"), (1, 1100, 16, 2, 64, "f32"), (20, 140, 32, 16, 128, "bf16"),
]


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d,dtype", CASES)
def test_forward_matches_the_token_loop(Bt, T, Hq, Hkv, d, dtype):
    _forward_case(Bt, T, Hq, Hkv, d, dtype, 3 + T)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32"), (64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -0.7, -3.0, -40.0, float("-inf")])
def test_forward_from_no_decay_to_no_memory(d, dtype, decay):
    _forward_case(2, 290, 4, 2, d, dtype, 11, decay=decay)


@pytest.mark.parametrize("d,dtype,G", [(128, "bf16", 1), (128, "bf16", 4), (64, "f32", 2), (64, "bf16", 1)])
@pytest.mark.parametrize("T,lens", [(300, [300, 0, 1, 128, 129, 255]), (130, [2, 130, 127, 0, 31, 64]),
                                     (700, [700, 1, 512, 513, -5, 9000])])
def test_forward_of_a_padded_batch(d, dtype, G, T, lens):
    q, k, v, ld, S, out, S1 = _forward_case(len(lens), T, 2 * G, 2, d, dtype, 5, lens=lens)
    for b, n in enumerate(lens):
        n = min(max(n, 0), T)
        assert not bool(out[b, n:].any())                 # padding rows are zeros, whatever the inputs hold there
        if n == 0:
            assert torch.equal(S1[b], S[b])               # and an empty sequence leaves its state bit for bit


def test_forward_without_a_state_and_with_a_scale():
    _forward_case(2, 200, 4, 2, 128, "bf16", 8, state=False, scale=0.37)
    _forward_case(2, 200, 4, 2, 64, "f32", 8, state=False, scale=2.5)


@pytest.mark.parametrize("Hq,Hkv,d,dtype", [(2, 2, 128, "bf16"), (8, 1, 128, "bf16"), (4, 4, 64, "f32"), (2, 1, 64, "bf16")])
def test_a_long_call_is_split_over_its_tokens_and_equals_its_parts(Hq, Hkv, d, dtype):
    # one sequence, few heads: the plan splits the token axis; two calls with the state handed on give the same
    T = 2500
    q, k, v, ld, S = _inputs(1, T, Hq, Hkv, d, dtype, 23)
    assert B.linear_scratch_bytes(1, T, Hq, Hkv, d, DT[dtype]) > 0
    out, S1 = B.linear_forward(q, k, v, ld, state=S)
    ref, rS = R.linear_forward(q, k, v, ld, S)
    mag, mS = R.linear_forward(q.abs(), k.abs(), v.abs(), ld, S.abs())
    _check("out", out, ref, mag, dtype, d + T + 64, tensor=True)
    _check("state", S1, rS, mS, "f32", d + T + 64)
    cut = 1111
    a, Sa = B.linear_forward(q[:, :cut].contiguous(), k[:, :cut].contiguous(), v[:, :cut].contiguous(), ld, state=S)
    b, Sb = B.linear_forward(q[:, cut:].contiguous(), k[:, cut:].contiguous(), v[:, cut:].contiguous(), ld, state=Sa, state_out=Sa)
    assert Sb.data_ptr() == Sa.data_ptr()
    _check("parts", torch.cat([a, b], 1), ref, mag, dtype, d + T + 64, tensor=True)
    _check("parts' state", Sb, rS, mS, "f32", d + T + 64)
    # in place, split: the first segment's state must not be overwritten before it is read
    S2 = S.clone()
    out2, S3 = B.linear_forward(q, k, v, ld, state=S2, state_out=S2)
    assert torch.equal(out2, out) and torch.equal(S3, S1)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("Bt,Hq,Hkv", [(1, 1, 1), (3, 8, 2), (2, 15, 1), (5, 24, 1), (37, 12, 4)])
def test_steps_match_the_token_loop(Bt, Hq, Hkv, d, dtype):
    T = 3
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, dtype, 31)
    ref, rS = R.linear_forward(q, k, v, ld, S)
    mag, mS = R.linear_forward(q.abs(), k.abs(), v.abs(), ld, S.abs())
    cur = S.clone()
    for t in range(T):
        x = [y[:, t].contiguous() for y in (q, k, v)]
        if t == 1:      # into a buffer of its own, the old state kept
            keep = cur.clone()
            out, nxt = B.linear_step(*x, ld, cur, state_out=torch.empty_like(cur))
            assert torch.equal(cur, keep)
            cur = nxt
        else:
            out, cur2 = B.linear_step(*x, ld, cur)
            assert cur2.data_ptr() == cur.data_ptr()
        _check("out %d" % t, out, ref[:, t], mag[:, t], dtype, d + 64)
    _check("state", cur, rS, mS, "f32", d + 64)


def test_a_prompt_then_steps_equal_one_call():
    q, k, v, ld, S = _inputs(2, 140, 4, 2, 128, "bf16", 41)
    out, S1 = B.linear_forward(q, k, v, ld, state=S)
    cut = 137
    a, cur = B.linear_forward(q[:, :cut].contiguous(), k[:, :cut].contiguous(), v[:, :cut].contiguous(), ld, state=S)
    rows = [a]
    for t in range(cut, 140):
        o, cur = B.linear_step(q[:, t].contiguous(), k[:, t].contiguous(), v[:, t].contiguous(), ld, cur)
        rows.append(o[:, None])
    mag, mS = R.linear_forward(q.abs(), k.abs(), v.abs(), ld, S.abs())
    got = torch.cat(rows, 1).double()
    assert ((got - out.double()).abs() <= 2 * (2.0 ** -8 * out.double().abs() + 2.0 ** -8 * mag)).all()
    assert ((cur.double() - S1.double()).abs() <= 600 * 2.0 ** -24 * mS).all()


def _magnitudes(d_out, q, k, v, ld, S, dS, lens):
    a = lambda x: None if x is None else torch.nan_to_num(x).abs()
    return R.linear_backward(a(d_out), a(q), a(k), a(v), ld, a(S), a(dS), lens)


def _backward_case(Bt, T, Hq, Hkv, d, dtype, seed, decay="spread", lens=None, state=True, d_state=True):
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, dtype, seed, decay, state)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    do = torch.randn(q.shape, generator=g, device="cuda").to(q.dtype)
    dS = torch.randn((Bt, Hkv, d, d), generator=g, device="cuda") if d_state else None
    lt = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if lens is not None:
        for b, n in enumerate(lens):
            for x in (q, k, v, do):
                x[b, n:] = float("nan")
    got = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS, lens=lt)
    torch.cuda.synchronize()
    zero = lambda x: torch.nan_to_num(x)
    ref = R.linear_backward(zero(do), zero(q), zero(k), zero(v), ld, S, dS, lens)
    mag = _magnitudes(do, q, k, v, ld, S, dS, lens)
    n = d + T * (Hq // Hkv) + 64
    for name, x, y, m in zip(("d_q", "d_k", "d_v"), got, ref, mag):
        _check(name, x, y, m, dtype, n, tensor=True)
    _check("d_state_in", got[3], ref[3], mag[3], "f32", n)
    return (do, q, k, v, ld, S, dS), got


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d,dtype", [
    (1, 1, 1, 1, 64, "f32"), (2, 1, 4, 2, 128, "bf16"), (2, 33, 2, 2, 64, "f32"), (1, 100, 6, 2, 128, "f32"),
    (1, 127, 2, 2, 128, "bf16"), (2, 128, 2, 1, 128, "bf16"), (1, 260, 8, 2, 128, "bf16"), (1, 300, 7, 1, 64, "bf16"),
    (1, 129, 3, 3, 64, "f32"), (1, 600, 2, 1, 128, "bf16"), (1, 520, 2, 2, 64, "f32"),
])
def test_backward_matches_automatic_differentiation(Bt, T, Hq, Hkv, d, dtype):
    _backward_case(Bt, T, Hq, Hkv, d, dtype, 7 + T)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32")])
@pytest.mark.parametrize("decay", [0.0, -0.9, -30.0, float("-inf")])
def test_backward_from_no_decay_to_no_memory(d, dtype, decay):
    _backward_case(1, 150, 4, 2, d, dtype, 13, decay=decay)


@pytest.mark.parametrize("d,dtype,G", [(128, "bf16", 1), (128, "bf16", 3), (64, "f32", 2), (64, "bf16", 1)])
def test_backward_of_a_padded_batch(d, dtype, G):
    lens = [150, 0, 1, 128, 129, 40]
    (do, q, k, v, ld, S, dS), got = _backward_case(len(lens), 150, 2 * G, 2, d, dtype, 17, lens=lens)
    for b, n in enumerate(lens):
        for x in got[:3]:
            assert not bool(x[b, n:].any())
    # an empty sequence hands its state's gradient through
    assert ((got[3][1] - dS[1]).abs() <= 2.0 ** -22 * dS[1].abs()).all()


def test_backward_without_state_or_its_gradient():
    _backward_case(1, 140, 2, 2, 128, "bf16", 19, state=False, d_state=False)
    _backward_case(1, 70, 2, 1, 64, "f32", 19, state=False, d_state=True)


def test_backward_agrees_with_differences_of_the_forward():
    # the loss is a polynomial in each input, so a central difference of the 64-bit forward is exact in q, and off by
    # O(h^2) terms elsewhere; h = 1e-4 leaves them below the fp32 error of the gradient
    q, k, v, ld, S = _inputs(1, 45, 4, 2, 64, "f32", 29)
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda x: torch.randn(x.shape, generator=g, device="cuda")
    do, dS = rnd(q), rnd(S)
    grads = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS)

    def loss(*x):
        o, s = R.linear_forward(x[0], x[1], x[2], ld, x[3])
        return float((o * do.double()).sum() + (s * dS.double()).sum())
    base = [x.double() for x in (q, k, v, S)]
    for i in range(4):
        dirn = rnd(base[i]).double()
        h = 1e-4
        hi, lo = list(base), list(base)
        hi[i], lo[i] = base[i] + h * dirn, base[i] - h * dirn
        num = (loss(*hi) - loss(*lo)) / (2 * h)
        ana = float((grads[i].double() * dirn).sum())
        size = float((grads[i].double() * dirn).abs().sum())
        assert abs(num - ana) <= 200 * 2.0 ** -24 * size + 1e-6 * size, (i, num, ana)


def test_the_same_call_gives_the_same_bits_and_masks_hold_special_values():
    q, k, v, ld, S = _inputs(3, 400, 4, 2, 128, "bf16", 37)
    lens = torch.tensor([400, 3, 200], dtype=torch.int32, device="cuda")
    for x in (q, k, v):
        x[1, 3:], x[2, 200:] = float("inf"), torch.finfo(x.dtype).min
    a = B.linear_forward(q, k, v, ld, state=S, lens=lens)
    b = B.linear_forward(q, k, v, ld, state=S, lens=lens)
    assert torch.isfinite(a[0].float()).all() and torch.isfinite(a[1]).all()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    do, dS = torch.randn_like(q.float()).to(q.dtype), torch.randn_like(S)
    c = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS, lens=lens)
    e = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS, lens=lens)
    assert all(torch.isfinite(x.float()).all() for x in c)
    assert all(torch.equal(x, y) for x, y in zip(c, e))


def test_calls_on_two_streams_and_in_a_replayed_graph_equal_the_plain_call():
    q, k, v, ld, S = _inputs(1, 1500, 2, 2, 128, "bf16", 43)
    do, dS = torch.randn_like(q.float()).to(q.dtype), torch.randn_like(S)
    ref = B.linear_forward(q, k, v, ld, state=S)
    refb = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for s in (s1, s2):
        with torch.cuda.stream(s):
            outs.append((B.linear_forward(q, k, v, ld, state=S), B.linear_backward(do, q, k, v, ld, state=S, d_state=dS)))
    torch.cuda.synchronize()
    for f, b in outs:
        assert all(torch.equal(x, y) for x, y in zip(f, ref)) and all(torch.equal(x, y) for x, y in zip(b, refb))
    # a captured step, prompt and backward, replayed on new values in the same buffers
    cur = S.clone()
    q1, k1, v1 = (x[:, 0].contiguous() for x in (q, k, v))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, _ = B.linear_step(q1, k1, v1, ld, cur)
        f = B.linear_forward(q, k, v, ld, state=S)
        b = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS)
    q.mul_(0.5)
    q1.copy_(q[:, 0])
    cur.copy_(S)
    g.replay()
    torch.cuda.synchronize()
    want, wS = B.linear_step(q1, k1, v1, ld, S, state_out=torch.empty_like(S))
    assert torch.equal(o, want) and torch.equal(cur, wS)
    assert all(torch.equal(x, y) for x, y in zip(f, B.linear_forward(q, k, v, ld, state=S)))
    assert all(torch.equal(x, y) for x, y in zip(b, B.linear_backward(do, q, k, v, ld, state=S, d_state=dS)))


def test_nothing_is_written_outside_the_outputs():
    # results in the middle of a larger buffer: the bands around them keep their bytes
    Bt, T, Hq, Hkv, d = 2, 131, 4, 2, 128
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, "bf16", 47)

    def banded(x):
        n, pad = x.numel() * x.element_size(), 4096
        raw = torch.full((n + 2 * pad,), 0xA5, dtype=torch.uint8, device="cuda")
        return raw, raw[pad:pad + n].view(x.dtype).view(x.shape)
    bands = {n: banded(x) for n, x in (("out", q), ("state", S), ("dq", q), ("dk", k), ("dv", v), ("ds", S))}
    B.linear_forward(q, k, v, ld, state=S, out=bands["out"][1], state_out=bands["state"][1])
    B.linear_backward(q, q, k, v, ld, state=S, d_state=S, out=tuple(bands[n][1] for n in ("dq", "dk", "dv", "ds")))
    torch.cuda.synchronize()
    for n, (raw, _) in bands.items():
        assert bool((raw[:4096] == 0xA5).all()) and bool((raw[-4096:] == 0xA5).all()), n
    want = B.linear_forward(q, k, v, ld, state=S)
    assert torch.equal(bands["out"][1], want[0]) and torch.equal(bands["state"][1], want[1])


def test_the_path_from_tokens_to_outputs_and_back():
    # projections -> norm and rotation -> linear attention -> and the gradients back to the projected q, k, v
    Bt, T, Hq, Hkv, d, dm = 2, 150, 4, 2, 128, 256
    g = torch.Generator(device="cuda").manual_seed(53)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = n(Bt, T, dm).to(torch.bfloat16)
    w = [(n(h * d, dm) * dm ** -0.5).to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    q0, k0, v0 = B.project_qkv(x, *w)
    q0, k0, v0 = q0.view(Bt, T, Hq, d), k0.view(Bt, T, Hkv, d), v0.view(Bt, T, Hkv, d)
    wq, wk = (1 + 0.2 * n(d)).to(torch.bfloat16), (1 + 0.2 * n(d)).to(torch.bfloat16)
    pos = torch.arange(T, device="cuda").repeat(Bt, 1)
    freq = 10000.0 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) / (d // 2))
    ld = -(2.0 ** (-8.0 * torch.arange(1, Hkv + 1, device="cuda") / Hkv)).float()
    q, k = B.norm_rotate(q0, k0, wq, wk, pos, freq)
    out, S = B.linear_forward(q, k, v0, ld)
    d_out = n(Bt, T, Hq, d).to(torch.bfloat16)
    d_q, d_k, d_v, _ = B.linear_backward(d_out, q, k, v0, ld)
    d_q0, d_k0, d_wq, d_wk = B.norm_rotate_backward(d_q, d_k, q0, k0, wq, wk, pos, freq)

    leaves = [y.double().requires_grad_() for y in (q0, k0, v0, wq, wk)]
    rq = R.norm_rotate(leaves[0], leaves[3], pos, freq, 1e-6, False)
    rk = R.norm_rotate(leaves[1], leaves[4], pos, freq, 1e-6, False)
    lam = torch.exp(ld.double())[None, :, None, None]
    St = torch.zeros(Bt, Hkv, d, d, dtype=torch.float64, device="cuda")
    rows = []
    for t in range(T):
        St = lam * St + rk[:, t, :, :, None] * leaves[2][:, t, :, None, :]
        rows.append(d ** -0.5 * torch.einsum("bhgi,bhij->bhgj", rq[:, t].reshape(Bt, Hkv, -1, d), St).reshape(Bt, Hq, d))
    ro = torch.stack(rows, 1)
    grads = torch.autograd.grad((ro * d_out.double()).sum(), leaves)
    # every stage rounds its bfloat16 results once (and its operands on the tensor path): five independent roundings of
    # at most 2^-8/sqrt(3) rms each on the longest way
    tol = (5 ** 0.5) * 2.0 ** -8 / 3 ** 0.5 * 1.5
    for name, a, b in zip(("out", "d_q", "d_k", "d_v", "d_w_q", "d_w_k"), (out, d_q0, d_k0, d_v, d_wq, d_wk),
                          (ro.detach(), *grads)):
        err = float((a.double() - b).square().mean().sqrt() / b.square().mean().sqrt())
        assert err <= tol, (name, err)


@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 128), (8, 2, 128), (2, 2, 64), (6, 2, 64)])
def test_float_states_of_a_bfloat16_call_are_float_sums(Hq, Hkv, d):
    # 16 tokens are one step of a tensor-core sum for each part a product is split into: at most four of them, each cut
    # off (not rounded) at 2^-23 of the partial sum, and a decay's power, one rounding of 2^-24, in front.
    q, k, v, ld, S = _inputs(3, 16, Hq, Hkv, d, "bf16", 59, decay=-0.11)
    _, S1 = B.linear_forward(q, k, v, ld)
    _, ref = R.linear_forward(q, k, v, ld)
    _, mag = R.linear_forward(q.abs(), k.abs(), v.abs(), ld)
    assert bool(((S1.double() - ref).abs() <= 4.5 * 2.0 ** -23 * mag).all())
    do = torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(60), device="cuda").to(q.dtype)
    got = B.linear_backward(do, q, k, v, ld)[3]
    ref = R.linear_backward(do, q, k, v, ld)[3]
    mag = R.linear_backward(do.abs(), q.abs(), k.abs(), v.abs(), ld)[3]
    G = Hq // Hkv       # the heads of a group follow one another in the sum; one product with the scale behind it
    assert bool(((got.double() - ref).abs() <= (4 * G + 1.5) * 2.0 ** -23 * mag).all())


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 2)])
def test_a_large_state_under_a_strong_decay(Hq, Hkv):
    # the state is 2^40 times what the tokens add and gone after a few of them: nothing of it may stay
    q, k, v, ld, S = _inputs(1, 130, Hq, Hkv, 128, "bf16", 61, decay=-2.0)
    S = S * 2.0 ** 40
    out, S1 = B.linear_forward(q, k, v, ld, state=S)
    ref, rS = R.linear_forward(q, k, v, ld, S)
    mag, mS = R.linear_forward(q.abs(), k.abs(), v.abs(), ld, S.abs())
    _check("out", out[:, 40:], ref[:, 40:], mag[:, 40:], "bf16", 128 + 130 + 64, tensor=True)
    _check("state", S1, rS, mS, "f32", 128 + 130 + 64)


def test_a_stream_argument_owns_what_the_call_allocates():
    # the stream is kept busy, and the current stream takes and overwrites all memory that the call could have let go
    q, k, v, ld, S = _inputs(1, 1500, 2, 2, 128, "bf16", 67)
    need = B.linear_scratch_bytes(1, 1500, 2, 2, 128, torch.bfloat16)
    assert need > 0
    do = torch.randn_like(q.float()).to(q.dtype)
    want, wantb = B.linear_forward(q, k, v, ld, state=S), B.linear_backward(do, q, k, v, ld, state=S)
    w = torch.ones(128, device="cuda", dtype=torch.bfloat16)
    pos, freq = torch.arange(1500, device="cuda")[None], torch.linspace(1.0, 0.01, 64, device="cuda", dtype=torch.float64)
    wantn = B.norm_rotate_backward(q, k, q, k, w, w, pos, freq)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    got = B.linear_forward(q, k, v, ld, state=S, stream=s)
    gotb = B.linear_backward(do, q, k, v, ld, state=S, stream=s)
    gotn = B.norm_rotate_backward(q, k, q, k, w, w, pos, freq, stream=s)
    held = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (need, 2 * need, need, 1 << 20, 1 << 21) for _ in range(3)]
    torch.cuda.synchronize()
    for a, b in ((got, want), (gotb, wantb), (gotn, wantn)):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    del held


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d,lens", [(2, 300, 8, 2, 128, None), (1, 1500, 16, 2, 128, None), (1, 700, 15, 1, 64, None),
                                                (3, 400, 6, 2, 64, [400, 0, 129]), (40, 130, 8, 4, 128, None), (1, 1, 2, 1, 128, None)])
def test_the_state_gradient_of_shared_heads_is_as_exact_as_one_heads(Bt, T, Hq, Hkv, d, lens):
    # A head's share is cut off at most 2^-23 of what it has come to at each of 3 * 8 steps of a chunk.  The tokens enter
    # in the order of their weights, so with these decays the sums of the squares of what has come to be is at most the
    # last's; chunks before decay.  In root mean square that is below 24 * 2^-24 of the state, whatever the heads.
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, "bf16", 71)
    g = torch.Generator(device="cuda").manual_seed(72)
    do = torch.randn(q.shape, generator=g, device="cuda").to(q.dtype)
    dS = torch.randn((Bt, Hkv, d, d), generator=g, device="cuda")
    lt = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    lam, G = torch.exp(ld.double())[:, None, None], Hq // Hkv
    for first in (None, dS):
        got = B.linear_backward(do, q, k, v, ld, state=S, d_state=first, lens=lt)
        for b in range(Bt):
            ref = torch.zeros((Hkv, d, d), dtype=torch.float64, device="cuda") if first is None else dS[b].double().clone()
            for t in reversed(range(T if lens is None else lens[b])):
                x, y = (z[b, t].double().view(Hkv, G, d) for z in (q, do))
                ref = lam * (ref + d ** -0.5 * torch.einsum("hgi,hgj->hij", x, y))
            err = float((got[3][b].double() - ref).norm())
            assert err <= 24 * 2.0 ** -24 * float(ref.norm()), (b, err / float(ref.norm()))
        again = B.linear_backward(do, q, k, v, ld, state=S, d_state=first, lens=lt)
        assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("Hq,Hkv,dtype", [(4, 2, "bf16"), (2, 2, "bf16"), (4, 2, "f32")])
def test_backward_without_the_state_gradient(Hq, Hkv, dtype):
    q, k, v, ld, S = _inputs(1, 700, Hq, Hkv, 128, dtype, 73)
    with_it = B.linear_backward(q, q, k, v, ld, state=S, d_state=S)
    without = B.linear_backward(q, q, k, v, ld, state=S, d_state=S, want_d_state=False)
    assert without[3] is None
    n = 128 + 700 * (Hq // Hkv) + 64
    ref, mag = R.linear_backward(q, q, k, v, ld, S, S), _magnitudes(q, q, k, v, ld, S, S, None)
    for name, x, y, r, m in zip(("d_q", "d_k", "d_v"), without, with_it, ref, mag):
        _check(name, x, r, m, dtype, n, tensor=True)
        _check(name, y, r, m, dtype, n, tensor=True)


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 128), (6, 2, 128), (10, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("T", [1, 60, 129, 250])
def test_reverse_scans_of_shared_heads_that_begin_with_a_padded_chunk(Hq, Hkv, d, T):
    # every head of the group brings a tile of its own whose padding rows are zeroed: against the formula, and the same bits
    # each time while every SM runs such a scan
    _backward_case(2, T, Hq, Hkv, d, "bf16", 79 + T)
    q, k, v, ld, S = _inputs(80, T, Hq, Hkv, d, "bf16", 83)
    lens = torch.randint(0, T + 1, (80,), generator=torch.Generator().manual_seed(T), dtype=torch.int32).cuda()
    first = B.linear_backward(q, q, k, v, ld, state=S, d_state=S, lens=lens)
    assert all(torch.isfinite(x.float()).all() for x in first)
    for _ in range(20):
        again = B.linear_backward(q, q, k, v, ld, state=S, d_state=S, lens=lens)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def _slow_state(b, c, log_decay, first, reverse):
    """sum_t lambda^(T-1-t) b_t^T c_t + lambda^T first, or lambda^(t+1) in reverse; b, c [T, H, d] -> [H, d, d], float64."""
    T = b.shape[0]
    t = torch.arange(T, device=b.device, dtype=torch.float64)
    w = torch.exp(f64(log_decay)[None, :] * (t + 1 if reverse else T - 1 - t)[:, None])
    S = torch.einsum("thi,thj->hij", b.double() * w[:, :, None], c.double())
    return S if first is None else S + torch.exp(T * f64(log_decay))[:, None, None] * first.double()


def f64(x):
    return x.double()


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d,split", [(5, 4096, 32, 32, 128, False), (5, 2000, 32, 32, 64, False), (20, 4096, 16, 8, 128, True),
                                                 (1, 40000, 2, 2, 128, True)])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -1e-3, -0.0107, -0.0109, -0.03])
def test_float_states_of_long_slow_sequences(Bt, T, Hq, Hkv, d, split, decay):
    # What the header says of them: off by less than 1e-6 in root mean square, whatever is kept and however long.  In a chunk
    # of 128 tokens 24 sums are cut off, by 2^-24 / 1.39 of what has come to be on average, which grows as the root of the
    # tokens: 24 * 2/3 * 2^-24 / 1.39 = 0.69e-6 of the chunk's share.  The chunks' shares are added with rounding: n chunks
    # add n roundings of 2^-24 / sqrt(3) at most of a sum that grows as the root of n, sqrt(n/2) 2^-24 / sqrt(3), which is
    # 0.14e-6 for 32 chunks.  (The last three decays are about where a chunk leaves a quarter of the state: one that stays under
    # the sums loses 24 * 2^-24 / 1.39 of half of it on average, as the sum grows, and 1 / (1 - 1/4) of that in all: 0.69e-6.)
    assert (B.linear_scratch_bytes(Bt, T, Hq, Hkv, d, torch.bfloat16) > 0) == split
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, "bf16", 89, decay=decay)
    do = torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(90), device="cuda").to(q.dtype)
    for first in (None, S):
        got = B.linear_forward(q, k, v, ld, state=first)[1]
        back = B.linear_backward(do, q, k, v, ld, d_state=first)[3]
        G = Hq // Hkv
        for b in {0, Bt - 1}:
            ref = _slow_state(k[b], v[b], ld, None if first is None else first[b], False)
            err = float((got[b].double() - ref).norm() / ref.norm())
            assert err <= 1e-6, ("state", first is None, err)
            ref = d ** -0.5 * _slow_state(q[b], do[b], ld.repeat_interleave(G), None, True).view(Hkv, G, d, d).sum(1)
            if first is not None:
                ref = ref + torch.exp(T * f64(ld))[:, None, None] * first[b].double()
            err = float((back[b].double() - ref).norm() / ref.norm())
            assert err <= 1e-6, ("d_state_in", first is None, err)


@pytest.mark.parametrize("decay", [0.0, -1e-4, -0.05])
@pytest.mark.parametrize("Hq,d", [(2, 128), (4, 128), (2, 64)])
@pytest.mark.parametrize("inf", [float("inf"), float("-inf")])
def test_an_infinity_in_the_state_stays_where_it_is(Hq, d, decay, inf):
    q, k, v, ld, S = _inputs(80, 400, Hq, 2, d, "bf16", 97, decay=decay)   # (enough heads that a call is not split)
    S[0, 1, 3, 5] = inf
    out, S1 = B.linear_forward(q, k, v, ld, state=S)
    want = torch.isinf(S)
    assert torch.equal(torch.isinf(S1), want) and float(S1[0, 1, 3, 5]) == inf and not bool(torch.isnan(S1).any())
    G = Hq // 2
    sees = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    sees[0, :, G:, 5] = q[0, :, G:, 3] != 0
    assert torch.equal(torch.isinf(out), sees)
    assert torch.equal(torch.sign(out[sees].float()), torch.sign(q[0, :, G:, 3][sees[0, :, G:, 5]].float()) * (1 if inf > 0 else -1))


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d", [(1, 3000, 8, 2, 128), (2, 700, 6, 2, 64), (40, 200, 8, 4, 128)])
def test_backward_without_the_state_gradient_keeps_to_its_scratch(Bt, T, Hq, Hkv, d):
    q, k, v, ld, S = _inputs(Bt, T, Hq, Hkv, d, "bf16", 101)
    need = B.linear_scratch_bytes(Bt, T, Hq, Hkv, d, torch.bfloat16, backward=True, want_d_state=False)
    want = B.linear_backward(q, q, k, v, ld, state=S, d_state=S, want_d_state=False)
    raw = torch.full((need + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    got = B.linear_backward(q, q, k, v, ld, state=S, d_state=S, want_d_state=False, scratch=raw[4096:4096 + need])
    assert got[3] is None and all(torch.equal(x, y) for x, y in zip(got[:3], want[:3]))
    assert bool((raw[:4096] == 0xA5).all()) and bool((raw[-4096:] == 0xA5).all())


@pytest.mark.parametrize("Hq,d", [(2, 128), (4, 128), (2, 64)])
@pytest.mark.parametrize("decay", [-0.3, -1.0, -9.0, float("-inf")])
def test_large_tokens_under_a_strong_decay(Hq, d, decay):
    # up to the stated range: results without the scale below 2^63
    q, k, v, ld, S = _inputs(2, 200, Hq, 2, d, "bf16", 103, decay=decay)
    do = torch.randn(q.shape, generator=torch.Generator(device="cuda").manual_seed(104), device="cuda").to(q.dtype)
    q, k, v, do, S = q * 2.0 ** 17, k * 2.0 ** 17, v * 2.0 ** 20, do * 2.0 ** 17, S * 2.0 ** 40
    out, S1 = B.linear_forward(q, k, v, ld, state=S)
    ref, rS = R.linear_forward(q, k, v, ld, S)
    mag, mS = R.linear_forward(q.abs(), k.abs(), v.abs(), ld, S.abs())
    assert 2.0 ** 55 < float(ref.abs().max()) * d ** 0.5 < 2.0 ** 63
    n = d + 200 * (Hq // 2) + 64
    _check("out", out, ref, mag, "bf16", n, tensor=True)
    _check("state", S1, rS, mS, "f32", n)
    dS = S * 2.0 ** -20        # (v has 2^20 more than do)
    got = B.linear_backward(do, q, k, v, ld, state=S, d_state=dS)
    ref, mag = R.linear_backward(do, q, k, v, ld, S, dS), _magnitudes(do, q, k, v, ld, S, dS, None)
    for name, x, y, m in zip(("d_q", "d_k", "d_v"), got, ref, mag):
        assert float(y.abs().max()) * d ** 0.5 < 2.0 ** 63
        _check(name, x, y, m, "bf16", n, tensor=True)
    _check("d_state_in", got[3], ref[3], mag[3], "f32", n)


@pytest.mark.parametrize("Hq,Hkv,d", [(16, 16, 128), (8, 4, 128), (4, 4, 64)])
@pytest.mark.parametrize("T,calls,decay", [(100, 60, -1e-4), (128, 40, -1e-3), (16, 300, -1e-4), (1, 300, -0.01), (200, 20, -1e-4)])
def test_float_states_handed_from_call_to_call(Hq, Hkv, d, T, calls, decay):
    # a prompt in pieces: what a call leaves in the state must not add up over the calls (the bound is that of one call; the
    # calls' roundings are n = `calls` of 2^-24 / sqrt(3) at most of a sum that grows as the root of n: below 0.43e-6)
    q, k, v, ld, S = _inputs(1, T * calls, Hq, Hkv, d, "bf16", 107, decay=decay)
    cur = S
    for i in range(calls):
        x = [y[:, i * T:(i + 1) * T].contiguous() for y in (q, k, v)]
        cur = B.linear_forward(*x, ld, state=cur)[1]
    ref = _slow_state(k[0], v[0], ld, S[0], False)
    assert float((cur[0].double() - ref).norm() / ref.norm()) <= 1e-6
