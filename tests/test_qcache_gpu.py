"""GPU parity of the 8-bit cache (bct_qcache_append / _attend / _evict) against its formulas in 64 bits.

Codes, scales, positions, lengths and moved weights are defined exactly: they are equal.

Tolerances of the attention.  With M = sum_j p_j |v_j| and S = scale sum_i |q_i k_i| (the largest of the call):
  - a score is an fp32 sum of d products, and goes through a few more roundings (scales, the cap, the change of base; fp32
    tanh to 2^-22): off by at most e = (d + 16) 2^-24 S, and by cap 2^-21 more under a cap; a probability is then off by
    2 e of itself at most (its own score and the sum), and by 2^-21 for the two exponentials;
  - sums over n slots: n 2^-24 each, of the probabilities and of the outputs;
  - bfloat16: a probability is rounded to 11 bits where it multiplies a value, 2^-11 (half a step of fp16), and the output
    once, 2^-8 |out|; float: two fp16 terms, 2^-22, and 2^-24 |out|.  Float queries are two terms as well, 2^-22 S;
  - fp16 ends at 2^-24, and probabilities enter it as 2^15 p with p = 1 the row's largest: each is off by 2^-25 / 2^15 in any
    case, which shows where the largest ones meet values of (nearly) zero.  The sum of the p being at least 1, that is
    2^-40 |v| for each slot, n 2^-40 max |v| at most.
"""
import pytest
import torch

from paper_2411_15785_b200 import binding as B
from paper_2411_15785_b200 import build as bld

import _qcache_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _built():
    bld.build()
    B.load()


def _tokens(Bt, T, H, d, dtype, seed, loud=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((Bt, T, H, d), generator=g, device="cuda")
    if loud:
        x = x * torch.exp(loud * torch.randn((Bt, T, H, 1), generator=g, device="cuda"))
    return x.to(DT[dtype])


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def _planes(cache):
    return tuple(getattr(cache, n) for n in R.NAMES)


def _same(cache, ref, held_only=True):
    """Every plane equal, up to the slots held (what stands behind them is no one's)."""
    torch.cuda.synchronize()
    got = {n: getattr(cache, n).cpu().numpy() for n in R.NAMES}
    assert (got["state"] == ref.state).all(), (got["state"], ref.state)
    for b in range(ref.B):
        n = int(ref.state[0, b])
        nb = -(-n // R.BLOCK)
        for p in "kv":
            a, r = got[p + "_scale"][b, :, :nb], getattr(ref, p + "_scale")[b, :, :nb]
            assert ((a == r) | ((a != a) & (r != r))).all(), (b, p, a, r)
            assert (got[p][b, :, :n] == getattr(ref, p)[b, :, :n]).all(), (b, p)
        assert (got["position"][b, :, :n] == ref.position[b, :, :n]).all(), b
        w, rw = got["weight"][b, :, :n], ref.weight[b, :, :n]
        assert ((w == rw) | ((w != w) & (rw != rw))).all(), b


def _check_attend(cache, ref, q, lens=None, scale=0.0, cap=0.0, **kw):
    before = cache.weight.double().cpu()
    out = cache.attend(q, lens=_i32(lens), scale=scale, score_cap=cap, **kw)
    torch.cuda.synchronize()
    want, added, M, S, V = ref.attend(torch.nan_to_num(q), lens, scale if scale > 0 else None, cap, device="cuda")
    d, n, rows = q.shape[3], ref.C, q.shape[1] * q.shape[2] // ref.H
    f32 = q.dtype == torch.float32
    e = (d + 16) * 2.0 ** -24 * S + (2.0 ** -22 * S if f32 else 0.0) + cap * 2.0 ** -21
    p_off = 2 * e + 2.0 ** -21 + n * 2.0 ** -24
    tol = (p_off + n * 2.0 ** -24 + (2.0 ** -22 if f32 else 2.0 ** -11)) * M + (2.0 ** -24 if f32 else 2.0 ** -8) * want.abs() + n * 2.0 ** -40 * V + 1e-30
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), float((got - want).abs().max()), float(((got - want).abs() / tol).max()))
    w = cache.weight.double().cpu() - before
    if not kw.get("accumulate", True):
        assert bool((w == 0).all())
        return out
    wtol = (p_off + rows * 2.0 ** -24) * added + 2.0 ** -23 * (before.abs() + added) + 1e-30
    for b in range(ref.B):
        m = int(ref.state[0, b])
        bad = (w[b, :, :m] - added[b, :, :m]).abs() > wtol[b, :, :m]
        assert not bool(bad.any()), (b, float((w[b, :, :m] - added[b, :, :m]).abs().max()))
    ref.weight[:] = cache.weight.cpu().numpy()      # the account goes on from what the library has
    return out


def _filled(Bt, Hkv, d, C, dtype, held, seed, loud=0.3, new=0):
    """A cache that holds `held` tokens of each sequence, and its reference."""
    cache = B.QuantCache(Bt, Hkv, d, C)
    ref = R.Ref(_planes(cache))
    T = max(max(held), 1)
    k, v = _tokens(Bt, T, Hkv, d, dtype, seed, loud), _tokens(Bt, T, Hkv, d, dtype, seed + 1, loud)
    for b, n in enumerate(held):
        k[b, n:], v[b, n:] = float("nan"), float("nan")       # padding holds whatever memory held
    cache.append(k, v, _i32(held))
    ref.append(k, v, held)
    return cache, ref


# ---- append -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32"), (64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("loud", [0.0, 1.5])
def test_append_in_pieces_writes_the_codes_of_the_definition(d, dtype, loud):
    cache = B.QuantCache(3, 2, d, 200)
    ref = R.Ref(_planes(cache))
    for i, T in enumerate([1, 1, 30, 1, 40, 7, 64, 1]):
        k, v = _tokens(3, T, 2, d, dtype, 10 * i, loud), _tokens(3, T, 2, d, dtype, 10 * i + 1, loud)
        lens = [T, T // 2, 0] if i % 2 else None
        if lens is not None:
            for b, n in enumerate(lens):
                k[b, n:], v[b, n:] = float("nan"), float("inf")
        cache.append(k, v, _i32(lens))
        ref.append(k, v, lens)
        _same(cache, ref)


@pytest.mark.parametrize("C", [1, 31, 32, 33, 70])
def test_tokens_without_a_free_slot_are_dropped_and_nothing_is_written_behind_a_head(C):
    band = torch.full((3, 1, C + 64, 64), 77, dtype=torch.int8, device="cuda")   # a head's plane with a band behind it
    cache = B.QuantCache(1, 1, 64, C)
    planes = list(_planes(cache))
    planes[0], planes[1] = band[0, :, :C][None], band[1, :, :C][None]
    cache = B.QuantCache(1, 1, 64, C, planes=planes)
    ref = R.Ref(_planes(cache))
    for i, T in enumerate([1, C + 5, 3]):
        k, v = _tokens(1, T, 1, 64, "bf16", i), _tokens(1, T, 1, 64, "bf16", i + 9)
        cache.append(k, v)
        ref.append(k, v)
        _same(cache, ref)
    assert cache.held.tolist() == [C] and cache.seen.tolist() == [C]
    assert bool((band[:2, :, C:] == 77).all()) and bool((band[2] == 77).all())


def test_rounding_is_to_the_nearest_with_ties_to_the_even_code():
    # amax 127 makes the scale 1; halves are ties, their neighbours are not
    x = torch.zeros((1, 32, 1, 64), device="cuda")
    x[0, 0, 0, 0] = 127.0
    h = torch.arange(63, device="cuda") + 0.5
    x[0, 1, 0, 1:] = h
    x[0, 2, 0, 1:] = -h
    up = torch.nextafter(h, torch.full_like(h, 1e9))
    dn = torch.nextafter(h, torch.zeros_like(h))
    x[0, 3, 0, 1:], x[0, 4, 0, 1:], x[0, 5, 0, 1:], x[0, 6, 0, 1:] = up, dn, -up, -dn
    cache = B.QuantCache(1, 1, 64, 32)
    ref = R.Ref(_planes(cache))
    cache.append(x, x * 0.37)
    ref.append(x, x * 0.37)
    _same(cache, ref)
    assert float(cache.k_scale[0, 0, 0]) == 1.0
    assert cache.k[0, 0, 1, 1:5].tolist() == [0, 2, 2, 4]


@pytest.mark.parametrize("size", [0.0, 1e-45, 3e-39, 1e-37, 1e30, 3.0e38])
def test_append_of_the_smallest_and_largest_magnitudes(size):
    cache = B.QuantCache(1, 2, 64, 96)
    ref = R.Ref(_planes(cache))
    for i, T in enumerate([5, 40, 10]):
        k = _tokens(1, T, 2, 64, "f32", i).clamp(-1, 1) * size
        v = _tokens(1, T, 2, 64, "f32", i + 3).clamp(-1, 1) * (size if i != 1 else 1.0)
        cache.append(k, v)
        ref.append(k, v)
        _same(cache, ref)


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_spoils_its_block_only(what):
    cache, ref = _filled(1, 2, 64, 128, "bf16", [40], 3)
    k, v = _tokens(1, 50, 2, 64, "bf16", 5), _tokens(1, 50, 2, 64, "bf16", 6)
    k[0, 30, 1, 7] = what                                      # slot 70: block 2 of head 1
    cache.append(k, v)
    torch.cuda.synchronize()
    s = cache.k_scale[0].cpu()
    assert bool(torch.isnan(s[1, 2])) and int(torch.isnan(s).sum()) == 1 and not bool(torch.isnan(cache.v_scale).any())
    ref.append(k, v)
    _same(cache, ref)
    out = cache.attend(_tokens(1, 1, 2, 64, "bf16", 7))
    assert bool(torch.isfinite(out[0, 0, 0]).all()) and bool(torch.isnan(out[0, 0, 1]).all())


@pytest.mark.parametrize("plane", ["k", "v"])
@pytest.mark.parametrize("T,Hq,dtype", [(3, 2, "bf16"), (30, 1, "bf16"), (40, 4, "bf16"), (60, 16, "bf16"), (70, 2, "f32"), (6, 1, "f32"),
                                        (180, 2, "bf16"), (200, 4, "bf16")])
def test_rows_that_do_not_see_a_spoilt_block_stay_clean(T, Hq, dtype, plane):
    held = 64 + min(T, 32) // 2                                # the last block is seen by the later half of the last tokens
    cache, ref = _filled(1, 1, 64, 300, dtype, [held], 3)
    clean = cache.attend(_tokens(1, T, Hq, 64, dtype, 7), accumulate=False)
    getattr(cache, plane + "_scale")[0, 0, 2] = float("nan")
    out = cache.attend(_tokens(1, T, Hq, 64, dtype, 7))
    sees = torch.clamp(held - T + 1 + torch.arange(T), min=0)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[0, sees.cuda() > 64]).all())
    assert torch.equal(out[0, sees.cuda() <= 64], clean[0, sees.cuda() <= 64])
    if plane == "v":
        # probabilities are of the keys alone: the weights are what they are without the spoilt block, within the file head's
        # bounds (not bit by bit: a row's sum is taken relative to the blocks' value scales on the tensor path)
        _, added, _, S, _ = ref.attend(_tokens(1, T, Hq, 64, dtype, 7), device="cuda")
        p_off = 2 * ((64 + 16 + 4) * 2.0 ** -24 * S) + 2.0 ** -21 + 300 * 2.0 ** -24
        w = cache.weight[0, 0, :held].double().cpu()
        assert bool(((w - added[0, 0, :held]).abs() <= (p_off + T * Hq * 2.0 ** -24 + 2.0 ** -23) * added[0, 0, :held]).all())


# ---- attention --------------------------------------------------------------------------------------------------

STEPS = [  # Bt, Hq, Hkv, d, dtype, C, held
    (1, 1, 1, 128, "bf16", 64, [1]), (1, 1, 1, 64, "f32", 33, [33]), (2, 4, 2, 128, "bf16", 100, [31, 100]),
    (3, 6, 2, 64, "bf16", 97, [32, 33, 0]), (2, 7, 1, 128, "f32", 300, [299, 64]), (2, 8, 1, 64, "bf16", 500, [500, 3]),
    (1, 9, 1, 128, "bf16", 129, [129]), (2, 16, 1, 128, "bf16", 260, [255, 256]), (1, 23, 1, 128, "bf16", 70, [65]),
    (1, 33, 1, 64, "bf16", 257, [250]), (2, 17, 1, 128, "f32", 95, [95, 64]), (5, 32, 8, 128, "bf16", 700, [700, 0, 1, 350, 699]),
    (70, 4, 2, 64, "f32", 40, [i % 41 for i in range(70)]), (300, 2, 1, 64, "bf16", 65, [(7 * i) % 66 for i in range(300)]),
    (1, 8, 8, 128, "bf16", 9001, [9001]), (2, 32, 32, 128, "bf16", 2048, [2048, 2000]),
]


@pytest.mark.parametrize("Bt,Hq,Hkv,d,dtype,C,held", STEPS)
def test_one_token_against_the_cache(Bt, Hq, Hkv, d, dtype, C, held):
    cache, ref = _filled(Bt, Hkv, d, C, dtype, held, 3)
    for seed in (20, 21):      # twice: the second adds to the weights of the first
        q = 1.5 * _tokens(Bt, 1, Hq, d, dtype, seed)
        out = _check_attend(cache, ref, q)
    for b, n in enumerate(held):
        if n == 0:
            assert bool((out[b] == 0).all())


TOKENS = [  # Bt, T, Hq, Hkv, d, dtype, C, held, lens
    (1, 2, 1, 1, 128, "bf16", 64, [2], None), (2, 5, 8, 2, 128, "bf16", 300, [300, 77], None),
    (2, 4, 4, 4, 64, "f32", 200, [4, 190], None), (3, 8, 4, 1, 128, "bf16", 150, [100, 150, 8], [8, 3, 0]),
    (2, 11, 6, 2, 64, "bf16", 99, [99, 40], [11, 1]), (2, 33, 2, 2, 128, "f32", 130, [130, 33], None),
    (2, 40, 4, 2, 128, "bf16", 333, [300, 40], [40, 17]), (1, 65, 8, 1, 64, "bf16", 200, [65], None),
    (2, 128, 4, 2, 128, "bf16", 128, [128, 128], None), (3, 129, 6, 2, 128, "bf16", 500, [129, 400, 500], [129, 100, 0]),
    (2, 150, 3, 1, 64, "f32", 400, [399, 150], [150, 31]), (1, 257, 2, 2, 64, "bf16", 257, [257], None),
    (2, 300, 8, 2, 128, "bf16", 700, [700, 511], None), (1, 512, 1, 1, 128, "bf16", 1024, [1000], None),
    (1, 513, 15, 3, 64, "bf16", 600, [513], None), (2, 64, 40, 1, 128, "bf16", 96, [96, 64], [64, 63]),
    (1, 1025, 4, 4, 128, "bf16", 1030, [1030], None),
]


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d,dtype,C,held,lens", TOKENS)
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_several_tokens_see_up_to_themselves(Bt, T, Hq, Hkv, d, dtype, C, held, lens, cap):
    cache, ref = _filled(Bt, Hkv, d, C, dtype, held, 5)
    q = 1.5 * _tokens(Bt, T, Hq, d, dtype, 30)
    if lens is not None:
        for b, n in enumerate(lens):
            q[b, n:] = float("nan")
    out = _check_attend(cache, ref, q, lens, cap=cap)
    if lens is not None:
        for b, n in enumerate(lens):
            assert bool((out[b, n:] == 0).all())


MANY = [  # the row counts where another kernel takes over, caches that are shared out, and batches that fill the device
    (2, 3, 8, 1, 128, "bf16", 150, [150, 70], [3, 1]), (2, 25, 1, 1, 128, "bf16", 150, [150, 25], None),
    (2, 24, 1, 1, 128, "f32", 150, [150, 25], None), (2, 16, 8, 1, 128, "bf16", 900, [900, 17], [16, 15]),
    (2, 32, 8, 2, 64, "bf16", 600, [600, 300], [32, 1]), (1, 30, 8, 1, 128, "bf16", 20000, [19999], None),
    (1, 3, 24, 3, 128, "bf16", 20000, [20000], None), (2, 32, 1, 1, 64, "bf16", 170, [170, 32], None),
    (2, 33, 1, 1, 64, "bf16", 170, [170, 33], [33, 9]), (3, 4, 16, 2, 128, "bf16", 300, [300, 129, 2], [4, 3, 1]),
    (2, 33, 1, 1, 64, "f32", 170, [170, 33], None), (2, 32, 2, 2, 128, "f32", 400, [400, 32], [32, 20]), (2, 300, 2, 1, 128, "bf16", 9000, [9000, 8191], [300, 299]),
    (37, 20, 4, 2, 64, "bf16", 700, [(53 * i) % 701 for i in range(37)], [i % 21 for i in range(37)]),
    (37, 9, 12, 4, 128, "bf16", 520, [(37 * i) % 521 for i in range(37)], [9 - i % 10 for i in range(37)]),
    (40, 70, 16, 4, 128, "bf16", 1000, [(211 * i) % 1001 for i in range(40)], [(11 * i) % 71 for i in range(40)]),
    (75, 512, 4, 1, 64, "bf16", 2048, [2048 - 29 * i for i in range(75)], [512 - 7 * i for i in range(75)]),
    (40, 520, 8, 2, 64, "bf16", 1793, [1793 - 31 * i for i in range(40)], [520 - 13 * i for i in range(40)]),
]


@pytest.mark.parametrize("Bt,T,Hq,Hkv,d,dtype,C,held,lens", MANY)
def test_several_tokens_at_the_counts_of_rows_where_kernels_change(Bt, T, Hq, Hkv, d, dtype, C, held, lens):
    test_several_tokens_see_up_to_themselves(Bt, T, Hq, Hkv, d, dtype, C, held, lens, 0.0)


def test_lengths_outside_the_call_count_as_its_ends():
    got = []
    for lens in ([-3, 9, 2], [0, 4, 2]):
        cache, _ = _filled(3, 2, 128, 100, "bf16", [10, 60, 33], 8)
        k, v, q = (_tokens(3, 4, h, 128, "bf16", 50 + i) for i, h in enumerate((2, 2, 8)))
        cache.append(k, v, _i32(lens))
        out = cache.attend(q, lens=_i32(lens))
        torch.cuda.synchronize()
        got.append([out, cache.weight] + list(_planes(cache)))
    assert got[0][-1][0].tolist() == [10, 64, 35]
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("lens", [[1, 1], [0, 1], [-1, 7]])
def test_single_tokens_of_a_padded_batch(lens):
    cache, ref = _filled(2, 2, 128, 100, "bf16", [40, 63], 8)
    out = _check_attend(cache, ref, _tokens(2, 1, 8, 128, "bf16", 9), lens)
    assert bool((out[0] == 0).all()) == (lens[0] < 1)
    before = cache.weight.clone()
    cache.attend(_tokens(2, 1, 8, 128, "bf16", 10), lens=_i32([0, 0]))
    assert torch.equal(cache.weight, before)


@pytest.mark.parametrize("T", [1, 6, 140])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f32")])
def test_rows_that_see_nothing_are_zero(T, d, dtype):
    cache, ref = _filled(3, 2, d, 200, dtype, [0, 3, 5], 5)
    q = _tokens(3, T, 4, d, dtype, 31)
    out = _check_attend(cache, ref, q)                          # more tokens than slots: the first see none
    for b, n in enumerate([0, 3, 5]):
        assert bool((out[b, :max(T - n, 0)] == 0).all())


@pytest.mark.parametrize("T", [1, 150])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_size,k_size,scale", [(1e-20, 1e20, 0.0), (1e18, 1e-19, 0.0), (1e-30, 1e-30, 1.0), (1.0, 1.0, 5.0),
                                                 (30.0, 1.0, 0.0)])
def test_magnitudes_of_queries_and_keys(T, dtype, q_size, k_size, scale):
    cache = B.QuantCache(2, 2, 128, 256)
    ref = R.Ref(_planes(cache))
    k, v = _tokens(2, 200, 2, 128, dtype, 1) * k_size, _tokens(2, 200, 2, 128, dtype, 2) * 1e-3
    v[:, 100:] *= 1e6                                            # blocks whose scales are far apart
    cache.append(k, v)
    ref.append(k, v)
    _check_attend(cache, ref, _tokens(2, T, 4, 128, dtype, 3) * q_size, scale=scale)


@pytest.mark.parametrize("T", [1, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_query_that_is_not_finite_spoils_its_own_row_only(T, dtype):
    cache, ref = _filled(1, 1, 128, 300, dtype, [290], 8)
    q = _tokens(1, T, 8, 128, dtype, 9)
    clean = cache.attend(q, accumulate=False)
    q[0, T // 2, 3, 5] = float("nan")
    q[0, T - 1, 6, 100] = float("inf")
    out = cache.attend(q, accumulate=False)
    bad = torch.zeros((T, 8), dtype=torch.bool, device="cuda")
    bad[T // 2, 3] = bad[T - 1, 6] = True
    assert bool(torch.isnan(out[0][bad]).all())
    assert torch.equal(out[0][~bad], clean[0][~bad])


@pytest.mark.parametrize("T", [1, 7, 180])
def test_the_same_call_gives_the_same_bits(T):
    got = []
    for _ in range(2):
        cache, _ = _filled(3, 2, 128, 2000, "bf16", [2000, 1311, 700], 8)
        q = _tokens(3, T, 8, 128, "bf16", 9)
        got.append((cache.attend(q).clone(), cache.weight.clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("T", [1, 5, 160])
def test_without_the_account_the_outputs_are_the_same_and_the_weights_stay(T):
    cache, ref = _filled(2, 2, 128, 600, "bf16", [600, 333], 8)
    q = _tokens(2, T, 8, 128, "bf16", 9)
    a = _check_attend(cache, ref, q, accumulate=False)
    b = _check_attend(cache, ref, q)
    assert torch.equal(a, b)


# ---- eviction ---------------------------------------------------------------------------------------------------

def _weigh(cache, ref, seed, ties=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = 3 * torch.rand(cache.weight.shape, generator=g, device="cuda") ** 4
    if ties:
        w = (w * 2).round() - 1.0        # few values, negative ones and zeros among them
    cache.weight.copy_(w)
    ref.weight[:] = w.cpu().numpy()


EVICT = [  # Bt, Hkv, d, C, held, keep, recent
    (1, 1, 64, 1, [1], 0, 0), (1, 1, 128, 2, [2], 1, 0), (1, 1, 128, 33, [33], 32, 5), (1, 1, 64, 33, [33], 32, 32),
    (2, 2, 128, 100, [100, 60], 60, 10), (3, 2, 64, 300, [300, 0, 129], 128, 128), (2, 1, 128, 300, [300, 299], 1, 1),
    (1, 2, 64, 500, [500], 0, 0), (2, 3, 128, 1024, [1024, 1000], 1023, 64), (1, 2, 128, 2100, [2100], 1001, 0),
    (1, 1, 64, 3000, [2999], 2900, 2900), (1, 1, 128, 45000, [45000], 44990, 100),
]


@pytest.mark.parametrize("Bt,Hkv,d,C,held,keep,recent", EVICT)
@pytest.mark.parametrize("ties", [False, True])
def test_evict_keeps_what_the_definition_keeps(Bt, Hkv, d, C, held, keep, recent, ties):
    cache, ref = _filled(Bt, Hkv, d, C, "bf16", held, 7, loud=0.8)
    _weigh(cache, ref, 3, ties)
    cache.evict(keep, recent)
    ref.evict(keep, recent)
    _same(cache, ref)


def test_evict_counts_a_nan_as_more_than_any_number_and_both_zeros_alike():
    cache, ref = _filled(1, 1, 64, 64, "bf16", [64], 7)
    w = torch.arange(64, device="cuda", dtype=torch.float32)
    w[3], w[10], w[20], w[21], w[40] = float("nan"), float("inf"), -0.0, 0.0, -5.0
    cache.weight[0, 0] = w
    ref.weight[0, 0] = w.cpu().numpy()
    cache.evict(61)        # 40, then 0 (slot 0), then slot 20: its -0 is the zero of slots 0 and 21
    ref.evict(61)
    _same(cache, ref)
    assert sorted(set(range(64)) - set(cache.position[0, 0, :61].tolist())) == [0, 20, 40]


def test_evict_to_the_capacity_and_below_what_is_held_changes_nothing():
    cache, ref = _filled(2, 2, 64, 100, "bf16", [100, 50], 7)
    cache.evict(100)
    _same(cache, ref)
    cache.evict(100, recent=100)
    _same(cache, ref)
    small, sref = _filled(2, 2, 64, 100, "bf16", [40, 50], 7)
    small.evict(50, recent=3)
    _same(small, sref)


# ---- a run of them together -------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,dtype,Hq", [(128, "bf16", 8), (64, "f32", 2)])
def test_a_bounded_decode_of_a_padded_batch(d, dtype, Hq):
    """Prompts, then single and drafted tokens, with room made in front of each append: what serving does."""
    Bt, Hkv, C = 3, 2, 96
    cache = B.QuantCache(Bt, Hkv, d, C)
    ref = R.Ref(_planes(cache))
    seed = 100
    for T, lens in [(50, [50, 20, 7]), (60, [60, 1, 33]), (1, None), (1, None), (4, [4, 2, 0]), (1, None), (40, None), (1, None),
                    (1, None)]:
        cache.evict(C - T, recent=min(8, C - T))
        ref.evict(C - T, recent=min(8, C - T))
        k, v, q = (_tokens(Bt, T, h, d, dtype, seed + i, 0.5) for i, h in enumerate((Hkv, Hkv, Hq)))
        seed += 3
        cache.append(k, v, _i32(lens))
        ref.append(k, v, lens)
        _same(cache, ref)
        _check_attend(cache, ref, q, lens)
    assert cache.seen.tolist() == ref.state[1].tolist()


def test_the_error_of_a_value_stays_below_one_step_however_it_was_written():
    """Token by token with rising magnitudes (the scale grows many times), then moved by evictions."""
    cache = B.QuantCache(1, 1, 64, 32)
    xs = []
    for t in range(32):
        x = _tokens(1, 1, 1, 64, "f32", t) * 1.35 ** t
        xs.append(x[0, 0, 0])
        cache.append(x, x)
    torch.cuda.synchronize()
    x = torch.stack(xs).double()
    s = float(cache.k_scale[0, 0, 0])
    assert 127.5 * s >= float(x.abs().max()) > 127.5 * s / 2
    err = (cache.k[0, 0].double() * s - x).abs()
    assert float(err.max()) < s
    assert float(err[-1].max()) <= 0.5 * s * (1 + 1e-9)


def test_a_captured_step_replays_with_the_lengths_of_the_moment():
    Bt, Hq, Hkv, d, C = 2, 4, 2, 128, 64
    cache, ref = _filled(Bt, Hkv, d, C, "bf16", [60, 30], 3)
    k, v, q = (_tokens(Bt, 1, h, d, "bf16", 50 + i) for i, h in enumerate((Hkv, Hkv, Hq)))
    out = torch.empty_like(q)

    def step():
        cache.evict(C - 1, recent=8)
        cache.append(k, v)
        cache.attend(q, out=out)

    planes = [t.clone() for t in _planes(cache)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    for t, p in zip(_planes(cache), planes):
        t.copy_(p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other = B.QuantCache(Bt, Hkv, d, C, planes=planes)
    for i in range(9):
        for x in (k, v, q):
            x.copy_(_tokens(*x.shape, "bf16", 60 + i))
        graph.replay()
        other.evict(C - 1, recent=8)
        other.append(k, v)
        want = other.attend(q)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for a, b in zip(_planes(cache), _planes(other)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("T,Hq,dtype", [(40, 8, "bf16"), (6, 8, "bf16"), (40, 8, "f32"), (150, 4, "bf16")])
def test_a_captured_prompt_replays_with_the_lengths_of_the_moment(T, Hq, dtype):
    Bt, Hkv, d, C = 3, 2, 64, 400
    cache, ref = _filled(Bt, Hkv, d, C, dtype, [390, 100, 0], 3)
    k, v, q = (_tokens(Bt, T, h, d, dtype, 50 + i) for i, h in enumerate((Hkv, Hkv, Hq)))
    lens, out = _i32([T, T // 2, 1]), torch.empty_like(q)

    def step():
        cache.evict(C - T, recent=20)
        cache.append(k, v, lens)
        cache.attend(q, lens, out=out, score_cap=20.0)

    planes = [t.clone() for t in _planes(cache)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    for t, p in zip(_planes(cache), planes):
        t.copy_(p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other = B.QuantCache(Bt, Hkv, d, C, planes=planes)
    for i in range(5):
        for x in (k, v, q):
            x.copy_(_tokens(*x.shape, dtype, 60 + i))
        lens.copy_(_i32([T - i, (T * i) // 4, 2 * i]))
        graph.replay()
        other.evict(C - T, recent=20)
        other.append(k, v, lens)
        want = other.attend(q, lens, score_cap=20.0)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for b, n in enumerate(cache.held.tolist()):
            for x, y in zip(_planes(cache)[:6], _planes(other)[:6]):
                m = -(-n // 32) if x.shape[2] != C else n
                assert torch.equal(x[b, :, :m], y[b, :, :m]), (i, b)
        assert torch.equal(cache.state, other.state)


@pytest.mark.parametrize("T,Hq,dtype", [(1, 2, "bf16"), (5, 4, "bf16"), (40, 4, "bf16"), (150, 8, "bf16"), (1, 2, "f32"), (40, 4, "f32")])
def test_what_memory_held_before_makes_no_difference(T, Hq, dtype):
    """Planes full of NaN, infinities and odd codes (but for the state): the calls go by what they have written."""
    Bt, Hkv, d, C = 3, 2, 64, 420
    clean = B.QuantCache(Bt, Hkv, d, C)
    planes = [t.clone() for t in _planes(clean)]
    planes[0].fill_(-128), planes[1].fill_(-77)
    planes[2].fill_(float("nan")), planes[3].fill_(float("inf")), planes[4].fill_(float("nan")), planes[5].fill_(0x7fffffff)
    dirty = B.QuantCache(Bt, Hkv, d, C, planes=planes)
    got = []
    for cache in (clean, dirty):
        outs = []
        for i, (n, lens) in enumerate([(T, [T, 0, 1]), (200, [200, 3, 64]), (T, None), (150, [10, 150, 33]), (T, None)]):
            k, v = (_tokens(Bt, n, Hkv, d, dtype, 90 + 3 * i + j, 0.4) for j in range(2))
            cache.evict(C - n, recent=8)
            cache.append(k, v, _i32(lens))
            outs.append(cache.attend(_tokens(Bt, n, Hq, d, dtype, 70 + i), _i32(lens)))
            outs.append(cache.attend(_tokens(Bt, T, Hq, d, dtype, 80 + i), accumulate=False))
        cache.evict(97, recent=5)
        outs.append(cache.attend(_tokens(Bt, T, Hq, d, dtype, 60)))
        got.append(outs)
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(*got)):
        assert bool(torch.isfinite(x).all()) and torch.equal(x, y), i
    assert torch.equal(clean.state, dirty.state)
    for b, n in enumerate(clean.held.tolist()):
        for x, y in zip(_planes(clean)[:6], _planes(dirty)[:6]):
            m = -(-n // 32) if x.shape[2] != C else n
            assert torch.equal(x[b, :, :m], y[b, :, :m]), b


@pytest.mark.parametrize("T", [1, 30])
def test_two_caches_at_once_on_two_streams(T):
    Bt, Hq, Hkv, d, C = 4, 8, 2, 128, 600

    def run(streams):
        caches = [_filled(Bt, Hkv, d, C, "bf16", [600, 400, 33, 500], 3 + i)[0] for i in range(2)]
        x = [[_tokens(Bt, T, h, d, "bf16", 80 + 3 * j + i) for i, h in enumerate((Hkv, Hkv, Hq))] for j in range(2)]
        torch.cuda.synchronize()
        outs = [[], []]
        for _ in range(12):
            for j, cache in enumerate(caches):
                with torch.cuda.stream(streams[j]):
                    cache.evict(C - T, recent=10)
                    cache.append(x[j][0], x[j][1])
                    outs[j].append(cache.attend(x[j][2]))
        torch.cuda.synchronize()
        return caches, outs

    one = torch.cuda.current_stream()
    (a, oa), (b, ob) = run([one, one]), run([torch.cuda.Stream(), torch.cuda.Stream()])
    for j in range(2):
        for x, y in zip(oa[j], ob[j]):
            assert torch.equal(x, y)
        for x, y in zip(_planes(a[j]), _planes(b[j])):
            assert torch.equal(x, y)


def test_calls_on_a_stream_of_their_own():
    cache, ref = _filled(2, 2, 64, 128, "bf16", [100, 90], 3)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    k, v, q = (_tokens(2, 3, 2, 64, "bf16", 70 + i) for i in range(3))
    torch.cuda.synchronize()
    cache.evict(90, recent=4, stream=s)
    cache.append(k, v, stream=s)
    out = cache.attend(q, stream=s)
    s.synchronize()
    ref.evict(90, recent=4)
    ref.append(k, v)
    _same_but_weight(cache, ref)
    want = ref.attend(q)[0]
    assert float((out.double().cpu() - want).abs().max()) < 0.05


def _same_but_weight(cache, ref):
    ref.weight[:] = cache.weight.cpu().numpy()
    _same(cache, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_whose_offsets_pass_32_bits(dtype):
    Hkv, d, C = 2, 128, (1 << 23) + 40                         # 2^31 codes and more to a plane
    held = C - 7
    cache = B.QuantCache(1, Hkv, d, C)
    g = torch.Generator(device="cuda").manual_seed(5)
    for x in (cache.k, cache.v):
        x.view(-1).random_(-127, 128, generator=g)
    for x in (cache.k_scale, cache.v_scale):
        x.uniform_(0.01, 0.02, generator=g)
    cache.position[:] = torch.arange(C, dtype=torch.int32, device="cuda")
    cache.state[:2] = held
    for T, Hq in ((1, 2), (3, 8), (20, 4)):
        cache.weight.zero_()
        q = 2.0 * _tokens(1, T, Hq, d, dtype, T)
        out = cache.attend(q).double()
        G = Hq // Hkv
        for h in range(Hkv):
            x = q[0, :, h * G:(h + 1) * G].double().reshape(T * G, d)
            lim = torch.repeat_interleave(held - T + 1 + torch.arange(T, device="cuda"), G)[:, None]
            n_at = 1 << 20

            def scores(at):
                n = min(n_at, held - at)
                of = torch.arange(at, at + n, device="cuda")
                s = x @ (cache.k[0, h, at:at + n].double() * cache.k_scale[0, h, of // 32].double()[:, None]).T * d ** -0.5
                return s.masked_fill(of[None, :] >= lim, float("-inf")), of

            m = torch.stack([scores(at)[0].amax(-1) for at in range(0, held, n_at)]).amax(0)[:, None]
            total, want, mag, wmax = 0.0, 0.0, 0.0, 0.0
            parts = []
            for at in range(0, held, n_at):
                s, of = scores(at)
                p = torch.exp(s - m)
                V = cache.v[0, h, at:at + len(of)].double() * cache.v_scale[0, h, of // 32].double()[:, None]
                total, want, mag = total + p.sum(-1, keepdim=True), want + p @ V, mag + p @ V.abs()
                parts.append((of, p))
            want, mag = want / total, mag / total
            got = out[0, :, h * G:(h + 1) * G].reshape(T * G, d)
            # scores are below 64 here: 144 * 2^-24 of that each; sums over a warp's run of blocks and over the runs' parts;
            # probabilities and the output as everywhere (the file's head)
            e = 2 * 144 * 2.0 ** -24 * 64 + 2.0 ** -21 + 2 * (C / 1024 + 4096) * 2.0 ** -24
            tol = (e + 2.0 ** -11) * mag + 2.0 ** -8 * want.abs() + C * 2.0 ** -40 * 2.6
            assert bool(((got - want).abs() <= tol).all()), (T, h, float((got - want).abs().max()))
            for of, p in parts[:1] + parts[-1:]:
                added = (p / total).sum(0)
                w = cache.weight[0, h, of].double()
                assert bool(((w - added).abs() <= (e + 80 * 2.0 ** -24) * added + 1e-30).all()), (T, h)
    cache.weight.uniform_(0, 1, generator=g)
    keep, recent = C - 100, 50
    gone = torch.sort(cache.weight[0, :, :held - recent], stable=True).indices[:, :held - keep].sort().values
    codes = cache.k.clone()
    cache.evict(keep, recent)
    torch.cuda.synchronize()
    for h in range(Hkv):
        left = torch.ones(held, dtype=torch.bool, device="cuda")
        left[gone[h]] = False
        assert torch.equal(cache.position[0, h, :keep].sort().values, torch.arange(held, dtype=torch.int32, device="cuda")[left])
        stay = left[:keep]
        moved = torch.zeros((keep + 31) // 32 * 32, dtype=torch.bool, device="cuda")
        moved[:keep] = ~stay
        quiet = ~moved.view(-1, 32).any(-1)
        of = torch.nonzero(quiet).flatten()[-3:]               # blocks without holes are as they were
        for blk in of.tolist():
            assert torch.equal(cache.k[0, h, 32 * blk:32 * blk + 32], codes[0, h, 32 * blk:32 * blk + 32])
    k = _tokens(1, 60, Hkv, d, dtype, 9)
    cache.append(k, k)
    torch.cuda.synchronize()
    assert cache.held.tolist() == [keep + 60] and cache.seen.tolist() == [held + 60]
    of = torch.arange(keep, keep + 60, device="cuda")
    for h in range(Hkv):
        s = cache.k_scale[0, h, of // 32].double()[:, None]
        assert bool(((cache.k[0, h, of].double() * s - k[0, :, h].double()).abs() <= 0.5 * s * (1 + 1e-6)).all())


def test_what_a_cache_knows_of_its_calls_is_bounded():
    cache, ref = _filled(1, 1, 64, 300, "bf16", [300], 3)
    for keep in range(299, 100, -1):
        cache.evict(keep)
        ref.evict(keep)
    _same(cache, ref)
    assert len(cache._known) <= 64


def test_binding_refuses_what_does_not_fit():
    cache = B.QuantCache(2, 2, 64, 64)
    k = _tokens(2, 3, 2, 64, "bf16", 1)
    with pytest.raises(ValueError):
        cache.append(k, k.float())
    with pytest.raises(ValueError):
        cache.append(k[:1], k[:1])
    with pytest.raises(ValueError):
        cache.append(k.transpose(1, 2), k.transpose(1, 2))
    with pytest.raises(ValueError):
        cache.append(k, k, lens=torch.tensor([1, 2], device="cuda"))
    with pytest.raises(ValueError):
        cache.append(k.cpu(), k.cpu())
    with pytest.raises(ValueError):
        cache.append(k.half(), k.half())
    with pytest.raises(B.BctError):
        cache.attend(_tokens(2, 3, 3, 64, "bf16", 1))
    with pytest.raises(B.BctError):
        cache.attend(k, score_cap=-1.0)
    with pytest.raises(B.BctError):
        cache.attend(k, out=k)
    with pytest.raises(B.BctError):
        cache.attend(k, scratch=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.BctError):
        cache.evict(65)
    with pytest.raises(B.BctError):
        cache.evict(10, recent=11)
    with pytest.raises(B.BctError):
        B.QuantCache(2, 2, 96, 64)
    with pytest.raises(ValueError):
        B.QuantCache(2, 2, 64, 64, device="cpu")
    with pytest.raises(ValueError):
        B.QuantCache(2, 2, 64, 64, planes=_planes(cache)[:6])
    with pytest.raises(ValueError):
        B.QuantCache(2, 2, 64, 65, planes=_planes(cache))
    torch.cuda.synchronize()
    assert cache.held.tolist() == [0, 0]
