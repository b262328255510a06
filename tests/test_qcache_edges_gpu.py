"""GPU tests of the 8-bit cache where its arithmetic can go wrong: roundings next to a half, scales at the end of float's
range, values of very unlike blocks, spoilt queries and their accounts of weight.  Codes and scales are equal to the 64-bit
form; other tolerances are derived beside the tests."""
import numpy as np
import pytest
import torch

from paper_2411_15785_b200 import binding as B
from paper_2411_15785_b200 import build as bld

import _qcache_ref as R
from test_qcache_gpu import _filled, _planes, _same, _tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    bld.build()
    B.load()


def _near(x, steps):
    """Floats `steps` representable numbers above x (positive, normal)."""
    return (np.asarray(x, np.float32).view(np.int32) + np.asarray(steps, np.int32)).view(np.float32)


# ---- moves: codes times a scale, rounded to another scale's codes ------------------------------------------------

def _moved(d, holes, code, f, s, seed):
    """A cache for each (code, f, s): an eviction leaves `holes` places in block 0, whose scale is s, and moves as many rows
    of block 1 there, whose scale is f and whose largest code is `code`.  Equal to the 64-bit form, or fails."""
    rng = np.random.default_rng(seed)
    units = len(code)
    held = 33 if holes == 1 else 64                      # (one slot alone is found in another way)
    k = np.zeros((2, units, 1, 64, d), np.int8)
    k[:, :, 0, :32] = rng.integers(-127, 128, (2, units, 32, d))
    c = np.asarray(code)[None, :, None, None]
    k[:, :, 0, 32:] = rng.integers(-c, c + 1, (2, units, 32, d))
    at = rng.integers(0, d // 2, (2, units, 32, 1))      # each row has the code and its negative somewhere
    np.put_along_axis(k[:, :, 0, 32:], at, np.broadcast_to(c, at.shape).astype(np.int8), -1)
    np.put_along_axis(k[:, :, 0, 32:], at + d // 2, np.broadcast_to(-c, at.shape).astype(np.int8), -1)
    scale = np.stack([np.asarray(s, np.float32), np.asarray(f, np.float32)], -1)[:, None]
    weight = np.full((units, 1, 64), 1.0, np.float32)
    for u in range(units):
        weight[u, 0, rng.permutation(32)[:holes]] = 0
        if held == 64:
            weight[u, 0, 32 + rng.permutation(32)[:32 - holes]] = 0
    state = np.stack([np.full(units, held), np.full(units, held), np.zeros(units)]).astype(np.int32)
    position = np.broadcast_to(np.arange(64, dtype=np.int32), (units, 1, 64)).copy()
    planes = [torch.from_numpy(x).cuda() for x in (k[0], k[1], scale, scale.copy(), weight, position, state)]
    cache = B.QuantCache(units, 1, d, 64, planes=planes)
    ref = R.Ref(planes)
    cache.evict(32)
    ref.evict(32)
    _same(cache, ref)
    assert int(cache.k[:, :, :32].min()) >= -127 and int(cache.v[:, :, :32].min()) >= -127


# code, scale of the source, scale of the destination.  The quotients are 127.5 (twice), 122.5000005, 127.4999994 and 116.5;
# fl(code f) fl(1 / s) is up to 127.5 2^-23 = 1.5e-5 away from them
HALVES = [(119, "0x1.26ac0ep+0", "0x1.1306fcp+0"), (27, "0x1.405020p+2", "0x1.0f52eep+0"),
          (101, "0x1.d00680p+0", "0x1.7e958ep+0"), (124, "0x1.1503ap+0", "0x1.0d68ecp+0"), (121, "0x1.ad238p+0", "0x1.bdb7p+0")]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("holes", [1, 2, 9, 31])
@pytest.mark.parametrize("power", [0, -40, 90])
def test_moved_codes_next_to_a_half_are_those_of_the_exact_quotient(d, holes, power):
    _moved(d, holes, [c for c, _, _ in HALVES], [float.fromhex(f) * 2.0 ** power for _, f, _ in HALVES],
           [float.fromhex(s) * 2.0 ** power for _, _, s in HALVES], 5 + holes)


@pytest.mark.parametrize("d,holes", [(64, 1), (64, 3), (128, 5)])
@pytest.mark.parametrize("power,most", [(0, 127), (-126, 6)])               # (the smallest scales, whose half is no float)
def test_moved_codes_aimed_at_halves(d, holes, power, most):
    rng = np.random.default_rng(17 + holes)
    units = 1500
    s = _near(np.float32(2.0 ** power), rng.integers(0, 1 << 23, units) | 1)
    code = rng.integers(1, most + 1, units)
    half = rng.integers(code, most + 1) + 0.5                               # (above the code: f is above s)
    f = _near((half * s.astype(np.float64) / code).astype(np.float32), rng.integers(-1, 2, units))
    _moved(d, holes, code, f, s, 23)


# ---- append: the CTAs of a sequence hand its length over ---------------------------------------------------------

def test_the_length_moves_on_once_whatever_the_ctas_of_a_sequence_have_to_do():
    """Many CTAs to a sequence, most of them without a block of their own, which take their tickets at once."""
    Bt, Hkv, d, T = 3, 64, 64, 640
    cache = B.QuantCache(Bt, Hkv, d, 4000)
    k = torch.ones((Bt, T, Hkv, d), dtype=torch.bfloat16, device="cuda")
    held = torch.zeros(Bt, dtype=torch.int32, device="cuda")
    for i in range(120):
        lens = torch.tensor([1, i % 3, 40 * (i % 2)], dtype=torch.int32, device="cuda")
        cache.append(k, k, lens)
        held += lens
    torch.cuda.synchronize()
    assert torch.equal(cache.held, held) and torch.equal(cache.seen, held) and not bool(cache.state[2].any())
    for b, n in enumerate(held.tolist()):
        assert bool((cache.k[b, :, :n] == 127).all()) and bool((cache.k[b, :, n:] == 0).all())
        assert torch.equal(cache.position[b, :, :n], torch.arange(n, dtype=torch.int32, device="cuda").expand(Hkv, n))


# ---- evictions of many sequences ---------------------------------------------------------------------------------

@pytest.mark.parametrize("Bt,C,n,ties", [(295, 200, 40, False), (296, 200, 1, True), (296, 200, 40, True), (298, 8192, 1, True),
                                         (298, 8193, 700, False)])
def test_evictions_where_the_selection_takes_other_ctas(Bt, C, n, ties):
    cache = B.QuantCache(Bt, 1, 64, C)
    g = torch.Generator(device="cuda").manual_seed(5)
    cache.k.random_(-127, 128, generator=g), cache.v.random_(-127, 128, generator=g)
    cache.k_scale.uniform_(0.5, 2.0, generator=g), cache.v_scale.uniform_(0.5, 2.0, generator=g)
    cache.weight.uniform_(0.0, 3.0, generator=g)
    if ties:
        cache.weight.round_()
    cache.position[:] = torch.arange(C, dtype=torch.int32, device="cuda").flip(0)
    cache.state[:2] = C
    cache.state[0, ::3] = C - n // 2
    ref = R.Ref(_planes(cache))
    cache.evict(C - n, recent=20)
    ref.evict(C - n, recent=20)
    _same(cache, ref)


# ---- append: the smallest scales, whose half is no float ---------------------------------------------------------

@pytest.mark.parametrize("d,T", [(64, 32), (128, 20)])
def test_appended_codes_at_halves_of_the_smallest_scales(d, T):
    rng = np.random.default_rng(3)
    heads = 40
    s = _near(np.float32(2.0 ** -126), rng.integers(1, 1 << 23, heads) | 1)          # odd multiples of 2^-149
    x = np.zeros((1, T, heads, d), np.float32)
    for h in range(heads):
        amax = np.float32(127 * s[h].astype(np.float64))
        mine = np.float64(np.float32(np.float64(amax) / 127))
        half = (rng.integers(0, 126, (T, d)) + 0.5) * mine                          # exact in 64 bits, no multiple of 2^-149
        x[0, :, h] = (np.rint(half * 2.0 ** 149) + rng.integers(-1, 2, (T, d))) * 2.0 ** -149 * rng.choice([-1, 1], (T, d))
        x[0, 0, h, 0] = amax
    k = torch.from_numpy(x).cuda()
    cache = B.QuantCache(1, heads, d, 96)
    ref = R.Ref(_planes(cache))
    cache.append(k, k.flip(1))
    ref.append(k, k.flip(1))
    _same(cache, ref)


# ---- attention: blocks that are far apart ------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Bt,Hkv,T,G", [(10, 8, 130, 1), (2, 1, 40, 1), (1, 2, 64, 4)])
def test_quiet_values_behind_a_loud_tile_keep_their_terms(Bt, Hkv, T, G, d):
    """One slot has a row's largest probability, and no value; all others 2^-26 of it.  Slots 0..127 are 60 times as loud as the
    rest, on other features.  A term is off by 2^-31 of the largest value that its tile's scales stand for at most, besides the
    roundings that are relative to the terms: 2^-11 of a probability, 2^-8 of an output, (d + 16) 2^-24 of a score of 18 for
    its own and the sum's, n 2^-24 for each of two sums and 2^-21 for the exponentials."""
    C = 128 * 11 + 50
    n = C - 3
    cache = B.QuantCache(Bt, Hkv, d, C)
    k, v = torch.zeros((2, Bt, n, Hkv, d), device="cuda")
    k[:, 200, :, 0] = 18.0                               # the others' scores are 0, its own 18
    v[:, :128, :, 1::2] = 60.0
    v[:, 128:, :, 0::2] = 1.0
    v[:, 200] = 0.0
    cache.append(k, v)
    q = torch.zeros((Bt, T, Hkv * G, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    ref = R.Ref(_planes(cache))
    want, added, M, S, _ = ref.attend(q, scale=1.0, device="cuda")
    out = cache.attend(q, scale=1.0).double().cpu()
    blocks = -(-n // 32)
    tile = torch.arange(n) // 32 // 4
    s = torch.nn.functional.pad(cache.v_scale[0, 0, :blocks].double().cpu(), (0, -blocks % 4)).view(-1, 4).amax(-1) * 127
    near = torch.cumsum(2.0 ** -31 * s[tile], 0)[n - T:n]            # of the slots that token i sees (1 / sum is below 1)
    p_off = 2 * (d + 16) * 2.0 ** -24 * S + 2.0 ** -21 + 2 * n * 2.0 ** -24
    tol = (p_off + 2.0 ** -11) * M + 2.0 ** -8 * want.abs() + near[None, :, None, None]
    assert float(want[..., 0].min()) > 4 * float(near.max())         # (losing them all would show)
    assert bool(((out - want).abs() <= tol).all()), float(((out - want).abs() / tol).max())


@pytest.mark.parametrize("T,dtype", [(1, "bf16"), (6, "bf16"), (40, "bf16"), (150, "bf16"), (1, "f32"), (40, "f32")])
@pytest.mark.parametrize("power", [-90, 103])
def test_values_at_the_ends_of_the_range(T, dtype, power):
    """Largest values of 2^-90, and of 2^112 by the 300 slots seen (with a little to spare)."""
    cache = B.QuantCache(2, 2, 64, 320)
    k, v = _tokens(2, 300, 2, 64, dtype, 1), _tokens(2, 300, 2, 64, "f32", 2)
    v = (v / v.abs().amax() * 2.0 ** power).to(k.dtype)
    cache.append(k, v)
    ref = R.Ref(_planes(cache))
    q = _tokens(2, T, 8, 64, dtype, 3)
    want, _, M, S, V = ref.attend(q, device="cuda")
    out = cache.attend(q).double().cpu()
    f32 = dtype == "f32"
    e = (64 + 16) * 2.0 ** -24 * S + (2.0 ** -22 * S if f32 else 0.0)
    p_off = 2 * e + 2.0 ** -21 + 2 * 300 * 2.0 ** -24
    tol = (p_off + (2.0 ** -22 if f32 else 2.0 ** -11)) * M + (2.0 ** -24 if f32 else 2.0 ** -8) * want.abs() + 300 * 2.0 ** -31 * V
    assert bool(((out - want).abs() <= tol).all()), float(((out - want).abs() / tol).max())


# ---- a query that is not finite, and the account of weight -------------------------------------------------------

@pytest.mark.parametrize("Bt,T,Hq,Hkv,C,dtype", [
    (2, 1, 8, 1, 300, "bf16"), (2, 1, 1, 1, 300, "f32"), (2, 6, 4, 1, 300, "bf16"), (2, 40, 2, 1, 300, "f32"),     # by stored scores / keys
    (2, 40, 4, 2, 300, "bf16"), (2, 300, 4, 1, 700, "bf16"), (75, 300, 1, 1, 2048, "bf16"),          # the tensor path's three forms
])
@pytest.mark.parametrize("what,cap", [(float("nan"), 0.0), (float("inf"), 0.0), (float("nan"), 20.0)])
def test_a_query_that_is_not_finite_gives_nan_to_the_slots_that_its_row_sees_and_no_others(Bt, T, Hq, Hkv, C, dtype, what, cap):
    held = C - 5
    q = _tokens(Bt, T, Hq, 64, dtype, 9)
    bad_q = q.clone()
    bad_q[0, T // 2, 0, 5] = what
    got = []
    for x in (q, bad_q):
        cache, _ = _filled(Bt, Hkv, 64, C, dtype, [held] * Bt, 8)
        cache.attend(x, score_cap=cap)
        got.append(cache.weight[:, :, :held])
    clean, bad = got
    seen = held - T + T // 2 + 1
    assert bool(torch.isnan(bad[0, 0, :seen]).all())
    assert torch.equal(bad[0, 0, seen:], clean[0, 0, seen:])
    assert torch.equal(bad[1:], clean[1:]) and torch.equal(bad[0, 1:], clean[0, 1:])
    assert bool(torch.isfinite(clean).all())
