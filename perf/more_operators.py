"""The operators of the 8-bit cache, as cases that can be measured: attention of T >= 1 tokens over a cache of int8 codes
with one scale per block of 32 slots and head, which adds each slot's attention weight to its account (``attend``); the
quantised append of tokens (``fill``); and the eviction of the slots with the least accumulated weight with the append
that takes their place (``turn``).

``own = False`` computes them in their plain form, elementary torch operations in 32 bits; ``own = True`` makes the calls
of ``paper_2411_15785_b200.binding`` that a program makes.  Codes, positions and lengths are whole numbers: scales and
roundings are defined exactly, so they come out equal bit for bit.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 32       # slots that share a scale


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of one sequence, grouped heads, an odd length: latency of a single-stream decode step
        dict(name="step_b1_c2048", op="attend", B=1, Hq=32, Hkv=8, d=128, dtype="bf16", C=2048, L=1999, T=1, len_seed=0, cap=0.0),
        # the decode batch of the 7B-like shape, every cache full: throughput
        dict(name="step_b64_c2048", op="attend", B=64, Hq=32, Hkv=32, d=128, dtype="bf16", C=2048, L=2048, T=1, len_seed=0, cap=0.0),
        # a decode batch of sequences of unlike lengths, grouped heads
        dict(name="step_ragged_b37_c16384", op="attend", B=37, Hq=32, Hkv=8, d=128, dtype="bf16", C=16384, L=16384, T=1,
             len_seed=7, cap=0.0),
        # one very long sequence: few rows, a long axis
        dict(name="step_b1_c131072", op="attend", B=1, Hq=32, Hkv=8, d=128, dtype="bf16", C=131072, L=131071, T=1, len_seed=0,
             cap=0.0),
        # float, head_dim 64, an odd batch and a capacity that is no multiple of a block
        dict(name="step_f32_b13_c1000", op="attend", B=13, Hq=12, Hkv=4, d=64, dtype="f32", C=1000, L=997, T=1, len_seed=3, cap=0.0),
        # a few drafted tokens verified at once, scores capped
        dict(name="verify_b16_t5_c4096", op="attend", B=16, Hq=32, Hkv=8, d=128, dtype="bf16", C=4096, L=4001, T=5, len_seed=0,
             cap=30.0),
        # a prompt over its own keys: the matrix products are the cost
        dict(name="prompt_b2_t2048", op="attend", B=2, Hq=32, Hkv=8, d=128, dtype="bf16", C=4096, L=2048, T=2048, len_seed=0, cap=0.0),
        # a padded batch of prompts behind what their caches hold, head_dim 64, capped, odd sizes
        dict(name="prompt_ragged_b5_t777", op="attend", B=5, Hq=8, Hkv=8, d=64, dtype="bf16", C=2500, L=2477, T=777, len_seed=5,
             cap=50.0),
        # the same in float
        dict(name="prompt_f32_b2_t333", op="attend", B=2, Hq=8, Hkv=2, d=64, dtype="f32", C=700, L=640, T=333, len_seed=0, cap=0.0),
        # a padded batch of prompts into caches that hold something already
        dict(name="fill_b8_t4096", op="fill", B=8, Hq=32, Hkv=8, d=128, dtype="bf16", C=8192, L=1000, T=4096, len_seed=11),
        # every decode step of full caches: one slot out, one token in
        dict(name="turn_b64_n1_c4096", op="turn", B=64, Hq=32, Hkv=8, d=128, dtype="bf16", C=4096, n=1, recent=512),
        # room for a block of tokens at a time
        dict(name="turn_b16_n500_c8192", op="turn", B=16, Hq=32, Hkv=8, d=128, dtype="bf16", C=8192, n=500, recent=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: batch, lengths, capacities and token counts spread over their logarithm, either type, either head
    size, shared and unshared heads.  No drawn case moves more bytes or computes more than the largest listed one."""
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["attend", "attend", "attend", "prompt", "fill", "turn"])
        Hkv = rng.choice([1, 2, 4, 8, 16, 32])
        Hq = Hkv * rng.choice([1, 1, 2, 3, 4, 7, 8])
        if Hq > 64:
            continue
        case = dict(op="attend" if op == "prompt" else op, B=_log_int(rng, 1, 96), Hq=Hq, Hkv=Hkv, d=rng.choice([64, 128, 128]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
        if op in ("attend", "prompt"):
            case["T"] = rng.choice([1, 1, 1, rng.randint(2, 8)]) if op == "attend" else _log_int(rng, 9, 2048)
            case["C"] = _log_int(rng, max(64, case["T"]), 131072 if op == "attend" else 8192)
            case["L"] = rng.choice([case["C"], rng.randint(case["T"], case["C"])])
            case["len_seed"] = rng.choice([0, rng.randrange(1, 1000)])
            case["cap"] = rng.choice([0.0, 0.0, 30.0])
            scores = case["B"] * Hq * case["T"] * case["C"]      # the plain form holds them all, in 32 bits
            planes = case["B"] * Hkv * case["C"] * case["d"]
            if scores > 2 ** 29 or planes > 2 ** 29:
                continue
            if case["dtype"] == "f32" and work(case)["flops"] > most["flops"] / 16:
                continue
        else:
            case["C"] = _log_int(rng, 64, 32768)
            if op == "fill":
                case["L"] = rng.randint(0, case["C"] - 1)
                case["T"] = _log_int(rng, 1, case["C"] - case["L"])
                case["len_seed"] = rng.choice([0, rng.randrange(1, 1000)])
            else:
                case["n"] = rng.choice([1, _log_int(rng, 1, case["C"] // 4)])
                case["recent"] = rng.randint(case["n"], case["C"] // 2)
            if case["B"] * Hkv * case["C"] * case["d"] > 2 ** 28:
                continue
        w = work(case)
        if all(w[k] <= most[k] for k in most):
            return case


def _lens(case):
    """For each sequence: (slots held before the pass, or seen by its last token for attend; new tokens of the padded
    batch)."""
    B, L = case["B"], case["L"]
    T = case.get("T", 1)
    if not case["len_seed"]:
        return [L] * B, [T] * B
    r = random.Random(case["len_seed"])
    if case["op"] == "fill":
        held = [r.randint(0, L) if i else L for i in range(B)]
        return held, [r.randint(0, T) if i else T for i in range(B)]
    seen = [r.randint(T, L) if i else L for i in range(B)]
    return seen, [r.randint(0, T) if i and T > 1 else T for i in range(B)]


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    B, Hq, Hkv, d, C = (case[k] for k in ("B", "Hq", "Hkv", "d", "C"))
    slot = 2 * d + 2 * 4 / BLOCK                  # codes and scales of a slot
    if case["op"] == "attend":
        seen, new = _lens(case)
        slots = sum(s for s, n in zip(seen, new) if n)
        pairs = sum(n * s - n * (n - 1) // 2 for s, n in zip(seen, new))
        # codes once, the weights' account read and written, queries in, outputs out
        return {"bytes": Hkv * slots * (slot + 8) + 2 * B * case["T"] * Hq * d * es, "flops": 4 * pairs * Hq * d}
    if case["op"] == "fill":
        n = sum(_lens(case)[1])
        return {"bytes": n * Hkv * (2 * d * es + slot + 8), "flops": 4 * n * Hkv * d}
    n, keep = case["n"], C - case["n"]
    moved = n * keep / C                          # evicted slots are spread over the cache: those below `keep` are filled again
    return {"bytes": B * Hkv * (8 * C + moved * (2 * slot + 16) + n * (2 * d * es + slot + 8)),
            "flops": B * Hkv * (2 * C + 4 * (n + moved) * d)}


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 23)
    dt = _dtype(case)
    B, Hq, Hkv, d, C = (case[k] for k in ("B", "Hq", "Hkv", "d", "C"))
    NB = -(-C // BLOCK)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def codes():
        c = torch.randn((B, Hkv, C, d), generator=g, device="cuda", dtype=torch.bfloat16).mul_(127 / 4)
        return c.round_().clamp_(-127, 127).to(torch.int8)

    st = dict(case=case, k=codes(), v=codes())
    st["k_scale"], st["v_scale"] = ((0.8 + 0.45 * rand(B, Hkv, NB)) * (4 / 127) for _ in range(2))
    # what attention has given each slot so far: little to most, much to a few
    st["weight"] = 3 * rand(B, Hkv, C) ** 4
    # earlier evictions have left the slots in some order, and have thinned out what was seen
    order = torch.argsort(rand(B, Hkv, C), dim=-1).int()
    st["position"] = 2 * order + torch.randint(0, 2, (B, Hkv, C), generator=g, device="cuda", dtype=torch.int32)
    if case["op"] == "attend":
        seen, new = _lens(case)
        st["q"] = 2 * normal(B, case["T"], Hq, d)
    else:
        seen, new = _lens(case) if case["op"] == "fill" else ([C] * B, [case["n"]] * B)
        n = case["T"] if case["op"] == "fill" else case["n"]
        loud = 1 + rand(B, n, Hkv, 1).to(dt)      # some tokens are louder than what their block has held
        st["new_k"], st["new_v"] = normal(B, n, Hkv, d) * loud, normal(B, n, Hkv, d) * loud
    ragged = case.get("len_seed", 0) != 0 and max(new) > 1
    st["lens"] = torch.tensor(new, dtype=torch.int32, device="cuda") if ragged else None
    # slots held, tokens seen, and a word of the library's own for each sequence
    state = [seen, [2 * C] * B, [0] * B]
    st["state"] = torch.tensor(state, dtype=torch.int32, device="cuda")
    if case["op"] == "fill":
        st["before"] = st["state"].clone()
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    if case["op"] == "fill":
        st["state"].copy_(st["before"])           # the caches as they were: the prompts go in again
    if own:
        return _run_own(case, st)
    if case["op"] == "attend":
        return _plain_attend(case, st)
    if case["op"] == "turn":
        _plain_evict(case, st)
    _plain_append(case, st)
    return _planes(st)


def _planes(st):
    return tuple(st[k] for k in ("k", "v", "k_scale", "v_scale", "weight", "position")) + (st["state"][:2],)


def _run_own(case, st):
    from paper_2411_15785_b200 import binding
    cache = st.get("cache")
    if cache is None:                             # the handle that a program keeps
        planes = tuple(st[k] for k in ("k", "v", "k_scale", "v_scale", "weight", "position", "state"))
        cache = st["cache"] = binding.QuantCache(case["B"], case["Hkv"], case["d"], case["C"], planes=planes)
    if case["op"] == "attend":
        out = cache.attend(st["q"], lens=st["lens"], score_cap=case["cap"])
        return out, st["weight"]
    if case["op"] == "turn":
        cache.evict(case["C"] - case["n"], recent=case["recent"])
    cache.append(st["new_k"], st["new_v"], lens=st["lens"])
    return _planes(st)


# ---- plain forms ------------------------------------------------------------------------------------------------

def _new_tokens(case, st, n):
    return torch.full((case["B"],), n, device="cuda") if st["lens"] is None else st["lens"].long()


def _values(codes, scale):
    """Codes [B, Hkv, C, d] as the values they stand for."""
    C = codes.shape[2]
    return codes.float() * scale.repeat_interleave(BLOCK, dim=2)[:, :, :C, None]


def _plain_attend(case, st):
    B, Hq, Hkv, d, C, T = (case[k] for k in ("B", "Hq", "Hkv", "d", "C", "T"))
    G = Hq // Hkv
    q = st["q"].float().view(B, T, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, d)
    s = torch.matmul(q, _values(st["k"], st["k_scale"]).transpose(-1, -2)).mul_(d ** -0.5)
    if case["cap"]:
        s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
    s = s.view(B, Hkv, G, T, C)
    n, i = _new_tokens(case, st, T)[:, None], torch.arange(T, device="cuda")
    sees = torch.where(i < n, st["state"][0][:, None] - n + i + 1, 0)             # [B, T] slots that a token sees
    hidden = torch.arange(C, device="cuda") >= sees[:, None, None, :, None]
    s.masked_fill_(hidden, float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == float("-inf"), 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))
    out = torch.matmul(p.view(B, Hkv, G * T, C), _values(st["v"], st["v_scale"]))
    out = out.view(B, Hkv, G, T, d).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, d)
    st["weight"].add_(p.sum((2, 3)))
    return out.to(st["q"].dtype), st["weight"]


def _grown(scale, amax, fresh):
    """The scale of a block that takes values up to `amax` besides what it holds (fresh: it holds nothing), and the
    power of two by which the scale of what it holds has grown.  In 64 bits: values next to a border decide."""
    start = torch.where(amax > 0, (amax.double() / 127).float().clamp(min=2.0 ** -126), 0.0)
    ratio = amax.double() / (127.5 * scale.double())
    m, e = torch.frexp(torch.where(ratio > 1, ratio, 1.0))
    e = torch.where(m > 0.5, e, e - 1)
    power = torch.ldexp(torch.ones_like(ratio), e)
    fresh = fresh | (scale == 0)
    return torch.where(fresh, start, (scale.double() * power).float()), torch.where(fresh, 1.0, power)


def _coded(x, scale):
    """round(x / scale) in -127..127, ties to the even code (x, scale: 64 bits)."""
    return torch.where(scale > 0, x / torch.where(scale > 0, scale, 1.0), 0.0).round().clamp(-127, 127)


def _plain_append(case, st):
    B, Hkv, d, C = (case[k] for k in ("B", "Hkv", "d", "C"))
    T = st["new_k"].shape[1]
    NB, W = -(-C // BLOCK), (T + BLOCK - 1) // BLOCK + 1      # blocks of a cache, blocks that T tokens touch at most
    held = st["state"][0].long()
    n = torch.minimum(_new_tokens(case, st, T), C - held)
    first = torch.clamp(held // BLOCK, max=NB - 1)
    block = first[:, None] + torch.arange(W, device="cuda")                                       # [B, W]
    slot = (block[:, :, None] * BLOCK + torch.arange(BLOCK, device="cuda")).view(B, W * BLOCK)    # [B, W * BLOCK]
    token = slot - held[:, None]
    is_new = (token >= 0) & (token < n[:, None])
    fresh = (block * BLOCK >= held[:, None])[:, None]
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None]
    # what has no place of its own goes where the first of its sequence goes, with the same values
    entry = torch.arange(W * BLOCK, device="cuda")
    entry = torch.where(slot < C, entry, 0)
    at = torch.gather(slot, 1, entry)[:, None]
    bentry = torch.where(block < NB, torch.arange(W, device="cuda"), 0)
    bat = torch.gather(block, 1, bentry)[:, None]
    pick = token.clamp(0, T - 1)
    touched = is_new.view(B, 1, W, BLOCK).any(-1)
    for codes, scale, x in ((st["k"], st["k_scale"], st["new_k"]), (st["v"], st["v_scale"], st["new_v"])):
        x = x.float()[torch.arange(B, device="cuda")[:, None], pick].permute(0, 2, 1, 3)          # [B, Hkv, W * BLOCK, d]
        x = torch.where(is_new[:, None, :, None], x, 0.0)
        amax = x.abs().amax(-1).view(B, Hkv, W, BLOCK).amax(-1)
        old = scale[b, h, bat]
        new, power = _grown(old, amax, fresh)
        new = torch.where(touched, new, old)
        power = torch.where(touched, power, 1.0).repeat_interleave(BLOCK, dim=2)[..., None]
        there = codes[b, h, at].double()
        c = _coded(x.double(), new.double().repeat_interleave(BLOCK, dim=2)[..., None])
        c = torch.where(is_new[:, None, :, None], c, (there / power).round())
        codes[b, h, at] = torch.gather(c, 2, entry[:, None, :, None].expand_as(c)).to(torch.int8)
        scale[b, h, bat] = torch.gather(new, 2, bentry[:, None].expand_as(new))
    for plane, fill in ((st["weight"], torch.zeros_like(token)), (st["position"], st["state"][1][:, None] + token)):
        val = torch.where(is_new[:, None], fill[:, None].to(plane.dtype), plane[b, h, at])
        plane[b, h, at] = torch.gather(val, 2, entry[:, None].expand_as(val))
    st["state"][:2] += n.int()


def _plain_evict(case, st):
    B, Hkv, d, C = (case[k] for k in ("B", "Hkv", "d", "C"))
    keep, NB = C - case["n"], -(-C // BLOCK)
    held, seen = st["state"][0].long()[:, None, None], st["state"][1][:, None, None]
    out = (held - keep).clamp(min=0)
    slot = torch.arange(C, device="cuda")
    worth = torch.where(st["position"] >= seen - case["recent"], float("inf"), st["weight"])
    worth = torch.where(slot < held, worth.double(), float("nan"))                # NaN sorts last: no slot at all
    rank = torch.argsort(torch.argsort(worth, dim=-1, stable=True), dim=-1)
    gone = rank < out
    hole, mover = gone & (slot < keep), ~gone & (slot >= keep) & (slot < held)
    M = min(keep, case["n"])
    dest = torch.where(hole, slot, C).sort(-1).values[..., :M]
    src = torch.where(mover, slot, C).sort(-1).values[..., :M]
    some = dest[..., :1] < C
    real = dest < C
    # what has no move of its own makes the first one again, or leaves slot 0 as it is
    dest = torch.where(real, dest, torch.where(some, dest[..., :1], 0))
    src = torch.where(real, src.clamp(max=C - 1), torch.where(some, src[..., :1].clamp(max=C - 1), 0))
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None]
    blk = dest // BLOCK
    start = torch.arange(NB, device="cuda") * BLOCK
    kept = (keep - start).clamp(0, BLOCK)
    holes = torch.zeros((B, Hkv, NB), device="cuda", dtype=torch.int64).scatter_add_(2, blk, real.long())
    for codes, scale in ((st["k"], st["k_scale"]), (st["v"], st["v_scale"])):
        x = codes[b, h, src].double() * scale[b, h, src // BLOCK].double()[..., None]
        amax = torch.zeros((B, Hkv, NB), device="cuda", dtype=torch.float64)
        amax.scatter_reduce_(2, blk, torch.where(real, x.abs().amax(-1), 0.0), "amax")
        new, power = _grown(scale, amax, (holes == kept) & (kept > 0))
        new, power = torch.where(holes > 0, new, scale), torch.where(holes > 0, power, 1.0)
        at = torch.where(slot < keep, power.repeat_interleave(BLOCK, dim=2)[..., :C], 1.0)[..., None]
        c = _coded(x, new[b, h, blk].double()[..., None])
        c = torch.where((real | some)[..., None], c, codes[b, h, dest].double())
        codes.copy_(torch.where(at > 1, (codes / at).round(), codes))
        codes[b, h, dest] = c.to(torch.int8)
        scale.copy_(new)
    for plane in (st["weight"], st["position"]):
        plane[b, h, dest] = plane[b, h, src]
    st["state"][0].clamp_(max=keep)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    """The formulas in 64 bits: attention sequence by sequence and head by head, the cache's changes unit by unit."""
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, st)
    units = case["B"] * case["Hkv"]
    moved = st["new_k"].numel() * 2 + (units * case["C"] * 8 if case["op"] == "turn" else 0)
    if moved > 2 ** 28 or units > 2048:
        return None
    c = {k: x.cpu().numpy() for k, x in st.items() if isinstance(x, torch.Tensor) and x.dtype != torch.bfloat16}
    x = {k: st[k].float().cpu().numpy().astype(np.float64) for k in ("new_k", "new_v")}
    for b in range(case["B"]):
        for h in range(case["Hkv"]):
            held, seen = int(c["state"][0, b]), int(c["state"][1, b])
            unit = {k: c[k][b, h] for k in ("k", "v", "k_scale", "v_scale", "weight", "position")}
            if case["op"] == "turn":
                held = _exact_evict(unit, held, seen, case["C"] - case["n"], case["recent"])
            n = x["new_k"].shape[1] if st["lens"] is None else int(c["lens"][b])
            n = min(n, case["C"] - held)
            where = np.arange(held, held + n)
            for p in ("k", "v"):
                _exact_write(unit[p], unit[p + "_scale"], where, x["new_" + p][b, :n, h], held)
            unit["weight"][where] = 0
            unit["position"][where] = seen + np.arange(n)
        c["state"][0, b], c["state"][1, b] = held + n, seen + n
    return tuple(torch.from_numpy(c[k]) for k in ("k", "v", "k_scale", "v_scale", "weight", "position")) + (
        torch.from_numpy(c["state"][:2]),)


def _exact_write(codes, scale, where, x, end):
    """Rows x into the slots `where` of one head's codes, whose slots from `end` on hold nothing that is kept."""
    for blk in np.unique(where // BLOCK):
        mine = where // BLOCK == blk
        rows, lo = where[mine], blk * BLOCK
        hi = min(lo + BLOCK, end)
        stay = np.setdiff1d(np.arange(lo, max(hi, lo)), rows)
        amax = np.abs(x[mine]).max()
        s = float(scale[blk])
        if len(stay) == 0 or s == 0:
            s = float(np.float32(max(amax / 127, 2.0 ** -126))) if amax > 0 else 0.0
        else:
            while amax > 127.5 * s:
                s *= 2
            codes[stay] = np.rint(codes[stay] * (float(scale[blk]) / s))
        scale[blk] = s
        codes[rows] = np.clip(np.rint(x[mine] / s), -127, 127) if s > 0 else 0


def _exact_evict(u, held, seen, keep, recent):
    if held <= keep:
        return held
    worth = np.where(u["position"][:held] >= seen - recent, np.inf, u["weight"][:held].astype(np.float64))
    gone = np.zeros(held, bool)
    gone[np.lexsort((np.arange(held), worth))[:held - keep]] = True
    dest = np.nonzero(gone[:keep])[0]
    src = keep + np.nonzero(~gone[keep:])[0]
    if len(dest):
        for p in ("k", "v"):
            x = u[p][src].astype(np.float64) * u[p + "_scale"][src // BLOCK].astype(np.float64)[:, None]
            _exact_write(u[p], u[p + "_scale"], dest, x, keep)
        for p in ("weight", "position"):
            u[p][dest] = u[p][src]
    return keep


def _exact_attend(case, st):
    B, Hq, Hkv, d, T = (case[k] for k in ("B", "Hq", "Hkv", "d", "T"))
    G = Hq // Hkv
    seen, new = _lens(case)
    out = torch.zeros((B, T, Hq, d), dtype=torch.float64, device="cuda")
    weight = st["weight"].double()
    for b in range(B):
        n, C = new[b], seen[b]
        if n == 0:
            continue
        mask = torch.ones((n, C), dtype=torch.bool, device="cuda").tril(C - n)
        blk = torch.arange(C, device="cuda") // BLOCK
        for h in range(Hkv):
            K = st["k"][b, h, :C].double() * st["k_scale"][b, h][blk].double()[:, None]
            V = st["v"][b, h, :C].double() * st["v_scale"][b, h][blk].double()[:, None]
            s = torch.einsum("tgd,cd->gtc", st["q"][b, :n, h * G:(h + 1) * G].double(), K) / math.sqrt(d)
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            p = torch.softmax(s.masked_fill(~mask, -math.inf), -1)
            out[b, :n, h * G:(h + 1) * G] = torch.einsum("gtc,cd->tgd", p, V)
            weight[b, h, :C] += p.sum((0, 1))
    return out, weight
