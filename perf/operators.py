"""The operators of the linear-attention path, as cases that can be measured: the norm and position rotation of
queries and keys for each head (forward, backward) and linear attention with a decay for each head (a prompt of T
tokens, a single token, the backward pass).

``own = False`` computes them in their plain form, elementary torch operations in 32 bits; ``own = True`` makes the
calls of ``paper_2411_15785_b200.binding`` that a program makes.
"""
import math
import random

import torch

own = False

CHUNK = 128      # tokens per chunk of the plain form
EPS = 1e-6
THETA = 10000.0


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of one sequence, grouped heads: latency of a single-stream decode step
        dict(name="step_b1", op="step", B=1, Hq=32, Hkv=8, d=128, dtype="bf16"),
        # a decode batch of the 7B-like shape: every state is read and written once
        dict(name="step_b64", op="step", B=64, Hq=32, Hkv=32, d=128, dtype="bf16"),
        # float, head_dim 64, an odd batch
        dict(name="step_f32_b37", op="step", B=37, Hq=12, Hkv=4, d=64, dtype="f32"),
        # one long prompt over 8 states: few rows, a long axis
        dict(name="prompt_b1_t16384", op="forward", B=1, Hq=32, Hkv=8, d=128, dtype="bf16", T=16384, len_seed=0),
        # the throughput case: the training / prefill forward of the 7B-like shape
        dict(name="prompt_b8_t4096", op="forward", B=8, Hq=32, Hkv=32, d=128, dtype="bf16", T=4096, len_seed=0),
        # a padded batch of prompts of unlike lengths
        dict(name="prompt_ragged_b13_t777", op="forward", B=13, Hq=32, Hkv=8, d=128, dtype="bf16", T=777, len_seed=5),
        # backward of a training step
        dict(name="train_b4_t4096", op="backward", B=4, Hq=32, Hkv=32, d=128, dtype="bf16", T=4096, len_seed=0),
        # backward in float, head_dim 64, odd length
        dict(name="train_f32_b2_t333", op="backward", B=2, Hq=8, Hkv=2, d=64, dtype="f32", T=333, len_seed=0),
        # norm + rotation of one decode batch: latency
        dict(name="rotate_n64", op="rotate", N=64, Hq=32, Hkv=8, d=128, dtype="bf16", rot=128, pairs="halves", far=131072),
        # ... of a prompt batch
        dict(name="rotate_n32768", op="rotate", N=32768, Hq=32, Hkv=8, d=128, dtype="bf16", rot=128, pairs="halves", far=8192),
        # ... in float, head_dim 64, part of the head rotated, neighbouring pairs, an odd count
        dict(name="rotate_f32_n1111", op="rotate", N=1111, Hq=8, Hkv=2, d=64, dtype="f32", rot=32, pairs="neighbours", far=1000000),
        # its backward in a training step
        dict(name="rotate_train_n16384", op="rotate_backward", N=16384, Hq=32, Hkv=32, d=128, dtype="bf16", rot=128,
             pairs="halves", far=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: batch, lengths and token counts spread over their logarithm, either type, either head size,
    shared and unshared heads.  No drawn case moves more bytes than the largest listed one."""
    cap = max(work(c)["bytes"] for c in listed())
    cap_f32 = cap // 16          # float runs on the CUDA cores: its products are the cost, not its bytes
    while True:
        op = rng.choice(["step", "forward", "forward", "backward", "rotate", "rotate_backward"])
        Hkv = rng.choice([1, 2, 4, 8, 16, 32])
        G = rng.choice([1, 1, 2, 3, 4, 7, 8])
        case = dict(op=op, Hq=Hkv * G, Hkv=Hkv, d=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "f32"]))
        if case["Hq"] > 64:
            continue
        if op in ("rotate", "rotate_backward"):
            case["N"] = _log_int(rng, 1, 32768)
            case["rot"] = rng.choice([case["d"], case["d"], case["d"] // 2])
            case["pairs"] = rng.choice(["halves", "neighbours"])
            case["far"] = _log_int(rng, 128, 1 << 20)
        elif op == "step":
            case["B"] = _log_int(rng, 1, 256)
        else:
            case["B"] = _log_int(rng, 1, 16)
            case["T"] = _log_int(rng, 1, 16384)
            case["len_seed"] = rng.choice([0, 0, rng.randrange(1, 1000)])
        bytes_ = work(case)["bytes"]
        if bytes_ <= (cap_f32 if case["dtype"] == "f32" and op in ("forward", "backward") else cap):
            return case


def _lens(case):
    """Valid tokens of each sequence (a padded batch), or None: all T."""
    if not case["len_seed"]:
        return None
    r = random.Random(case["len_seed"])
    return [r.randint(0, case["T"]) if i else case["T"] for i in range(case["B"])]


def _tokens(case):
    lens = _lens(case)
    return case["B"] * case["T"] if lens is None else sum(lens)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    if case["op"] in ("rotate", "rotate_backward"):
        vec = case["N"] * (Hq + Hkv) * d
        io = case["N"] * 8 + 2 * d * es + case["rot"] // 2 * 8
        if case["op"] == "rotate":
            return {"bytes": 2 * vec * es + io, "flops": 8 * vec}
        return {"bytes": 3 * vec * es + io + 2 * d * 4, "flops": 16 * vec}
    state = case["B"] * Hkv * d * d * 4
    if case["op"] == "step":
        n = case["B"]
        return {"bytes": 2 * state + n * (2 * Hq + 2 * Hkv) * d * es, "flops": 2 * n * d * d * (Hkv + Hq)}
    n = _tokens(case)
    # the recurrence itself: a rank-one update per kv-head and token, a vector-matrix product per query head and token
    fwd = 2 * n * d * d * (Hkv + Hq)
    if case["op"] == "forward":
        return {"bytes": 2 * state + n * (2 * Hq + 2 * Hkv) * d * es, "flops": fwd}
    # backward: S forward and dS in reverse (two updates), and the products that give dq, dk and dv
    return {"bytes": 3 * state + n * (3 * Hq + 4 * Hkv) * d * es, "flops": 2 * n * d * d * (3 * Hkv + 2 * Hq)}


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    dt = _dtype(case)
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]

    def normal(*shape, std=1.0, dtype=dt):
        x = torch.randn(shape, generator=g, device="cuda", dtype=dtype)
        return x.mul_(std) if std != 1.0 else x

    st = dict(case=case)
    if case["op"] in ("rotate", "rotate_backward"):
        N = case["N"]
        st["q"], st["k"] = normal(N, Hq, d), normal(N, Hkv, d)
        st["w_q"] = (1.0 + 0.2 * normal(d, dtype=torch.float32)).to(dt)
        st["w_k"] = (1.0 + 0.2 * normal(d, dtype=torch.float32)).to(dt)
        st["positions"] = torch.randint(0, case["far"], (N,), generator=g, device="cuda", dtype=torch.int64)
        half = case["rot"] // 2
        st["freq"] = THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        if case["op"] == "rotate_backward":
            st["d_q"], st["d_k"] = normal(N, Hq, d), normal(N, Hkv, d)
        return st
    B = case["B"]
    # decays of the heads spread geometrically, as trained models fix them: the first head forgets within a few
    # tokens, the last keeps hundreds
    slopes = 2.0 ** (-8.0 * torch.arange(1, Hkv + 1, device="cuda", dtype=torch.float64) / Hkv)
    st["log_decay"] = (-slopes).float()
    st["state"] = normal(B, Hkv, d, d, dtype=torch.float32)
    if case["op"] == "step":
        st["q"], st["k"], st["v"] = normal(B, Hq, d), normal(B, Hkv, d), normal(B, Hkv, d)
        st["state_out"] = torch.empty_like(st["state"])     # a program that can step back keeps both
        return st
    T = case["T"]
    st["q"], st["k"], st["v"] = normal(B, T, Hq, d), normal(B, T, Hkv, d), normal(B, T, Hkv, d)
    lens = _lens(case)
    st["lens"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["op"] == "backward":
        st["d_out"] = normal(B, T, Hq, d)
        st["d_state"] = normal(B, Hkv, d, d, dtype=torch.float32)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    return (_run_own if own else _run_plain)(case["op"], case, st)


def _run_own(op, case, st):
    from paper_2411_15785_b200 import binding as B
    if op == "step":
        return B.linear_step(st["q"], st["k"], st["v"], st["log_decay"], st["state"], state_out=st["state_out"])
    if op == "forward":
        return B.linear_forward(st["q"], st["k"], st["v"], st["log_decay"], state=st["state"], lens=st["lens"])
    if op == "backward":
        return B.linear_backward(st["d_out"], st["q"], st["k"], st["v"], st["log_decay"], state=st["state"],
                                 d_state=st["d_state"], lens=st["lens"])
    inter = case["pairs"] == "neighbours"
    if op == "rotate":
        return B.norm_rotate(st["q"], st["k"], st["w_q"], st["w_k"], st["positions"], st["freq"], eps=EPS, interleaved=inter)
    return B.norm_rotate_backward(st["d_q"], st["d_k"], st["q"], st["k"], st["w_q"], st["w_k"], st["positions"], st["freq"],
                                  eps=EPS, interleaved=inter)


def _run_plain(op, case, st):
    if op == "step":
        return _plain_step(case, st)
    if op == "forward":
        return _plain_forward(case, st)
    if op == "backward":
        return _plain_backward(case, st)
    if op == "rotate":
        return _plain_rotate(case, st)
    return _plain_rotate_backward(case, st)


# ---- plain forms: linear attention ------------------------------------------------------------------------------

def _plain_step(case, st):
    B, Hq, Hkv, d = case["B"], case["Hq"], case["Hkv"], case["d"]
    q = st["q"].float().view(B, Hkv, Hq // Hkv, d) * d ** -0.5
    k, v = st["k"].float(), st["v"].float()
    s = st["state"] * torch.exp(st["log_decay"])[:, None, None] + k[..., :, None] * v[..., None, :]
    out = torch.matmul(q, s).reshape(B, Hq, d).to(st["q"].dtype)
    st["state_out"].copy_(s)
    return out, st["state_out"]


def _heads_first(x, Hkv, keep):
    """[B, T, H, d] -> float [B, Hkv, H/Hkv, T, d], rows that are padding set to zero."""
    B, T, H, d = x.shape
    x = x.float()
    if keep is not None:
        x = torch.where(keep[:, :, None, None], x, torch.zeros((), device=x.device))
    return x.view(B, T, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4)


def _heads_back(x, dtype):
    B, Hkv, G, T, d = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(B, T, Hkv * G, d).to(dtype)


def _keep(case, st):
    if st["lens"] is None:
        return None, torch.full((case["B"],), case["T"], device="cuda", dtype=torch.int64)
    lens = st["lens"].long()
    return torch.arange(case["T"], device="cuda")[None, :] < lens[:, None], lens


def _scan(a, b, c, log_decay, state, lens, reverse):
    """out_i = sum_j lambda^|i-j| (a_i . b_j) c_j over j <= i (reverse: j >= i), plus the state's share; a, b, c
    [B, Hkv, Ga | Gb | Gb, T, d], chunk by chunk.  Forward: the state before the chunk is seen with lambda^(i+1);
    reverse: the state behind the chunk's last valid row n-1 is seen with lambda^(n-1-i).
    Returns out [B, Hkv, Ga, T, d] (summed over b's heads) and the state after all chunks."""
    T = a.shape[3]
    g = log_decay[None, :, None]                                    # [1, Hkv, 1]
    out = torch.empty_like(a)
    starts = list(range(0, T, CHUNK))
    for s in reversed(starts) if reverse else starts:
        n = min(CHUNK, T - s)
        ac, bc, cc = a[:, :, :, s:s + n], b[:, :, :, s:s + n], c[:, :, :, s:s + n]
        i = torch.arange(n, device=a.device, dtype=torch.float32)
        valid = (lens - s).clamp(0, n).float()[:, None, None]       # [B, 1, 1] valid rows of this chunk
        dist = i[:, None] - i[None, :]
        if reverse:
            dist = -dist
        decay = torch.where(dist >= 0, torch.exp(dist.clamp(min=0) * log_decay[:, None, None]), torch.zeros((), device=a.device))
        to_end = torch.exp((valid - 1 - i).clamp(min=0) * g)        # [B, Hkv, n]
        from_start = torch.exp((i + 1) * g).expand_as(to_end)
        seen, added = (to_end, from_start) if reverse else (from_start, to_end)
        o = torch.matmul(ac, state[:, :, None]) * seen[:, :, None, :, None]
        for h in range(b.shape[2]):
            o = o + torch.matmul(torch.matmul(ac, bc[:, :, h:h + 1].transpose(-1, -2)) * decay[None, :, None], cc[:, :, h:h + 1])
        out[:, :, :, s:s + n] = o
        state = state * torch.exp(valid * g)[..., None]
        for h in range(b.shape[2]):
            state = state + torch.matmul((bc[:, :, h] * added[..., None]).transpose(-1, -2), cc[:, :, h])
    return out, state


def _plain_forward(case, st):
    Hkv, scale = case["Hkv"], case["d"] ** -0.5
    keep, lens = _keep(case, st)
    q, k, v = (_heads_first(st[n], Hkv, keep) for n in ("q", "k", "v"))
    out, state = _scan(q * scale, k, v, st["log_decay"], st["state"], lens, False)
    out = _heads_back(out, st["q"].dtype)
    if keep is not None:
        out = out.masked_fill(~keep[:, :, None, None], 0)
    return out, state


def _plain_backward(case, st):
    Hkv, scale, dt = case["Hkv"], case["d"] ** -0.5, st["q"].dtype
    keep, lens = _keep(case, st)
    q, k, v, do = (_heads_first(st[n], Hkv, keep) for n in ("q", "k", "v", "d_out"))
    ld = st["log_decay"]
    # the state that each pass carries has b's features in its rows and c's in its columns
    d_q, _ = _scan(do, v, k, ld, st["state"].transpose(-1, -2), lens, False)
    d_k, _ = _scan(v, do, q * scale, ld, st["d_state"].transpose(-1, -2), lens, True)
    d_v, d_s = _scan(k, q * scale, do, ld, st["d_state"], lens, True)
    outs = [_heads_back(x, dt) for x in (d_q * scale, d_k, d_v)]
    if keep is not None:
        outs = [x.masked_fill(~keep[:, :, None, None], 0) for x in outs]
    return (*outs, d_s)


# ---- plain forms: norm and rotation -----------------------------------------------------------------------------

def _turn(st):
    angle = st["positions"].double()[:, None, None] * st["freq"]    # far positions: the angle in 64 bits
    return torch.cos(angle).float(), torch.sin(angle).float()


def _halves(x, rot, inter):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])


def _rotated(x, cos, sin, rot, inter):
    y = x.clone()
    a, b = _halves(x, rot, inter)
    ya, yb = _halves(y, rot, inter)
    ya.copy_(a * cos - b * sin)
    yb.copy_(a * sin + b * cos)
    return y


def _plain_rotate(case, st):
    cos, sin = _turn(st)
    outs = []
    for x, w in ((st["q"], st["w_q"]), (st["k"], st["w_k"])):
        f = x.float()
        y = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * w.float()
        outs.append(_rotated(y, cos, sin, case["rot"], case["pairs"] == "neighbours").to(x.dtype))
    return tuple(outs)


def _plain_rotate_backward(case, st):
    cos, sin = _turn(st)
    dxs, dws = [], []
    for x, w, dy in ((st["q"], st["w_q"], st["d_q"]), (st["k"], st["w_k"], st["d_k"])):
        f = x.float()
        g = _rotated(dy.float(), cos, -sin, case["rot"], case["pairs"] == "neighbours")
        r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
        xh = f * r
        dws.append((g * xh).sum((0, 1), dtype=torch.float64).float())
        h = g * w.float()
        dxs.append((r * (h - xh * (h * xh).mean(-1, keepdim=True))).to(x.dtype))
    return (*dxs, *dws)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    """The recurrences token by token, and the norm's and rotation's formulas, in 64 bits."""
    st = prepare(case, seed)
    if case["op"] in ("rotate", "rotate_backward"):
        return _exact_rotation(case, st)
    if case["op"] == "step":
        one = {n: st[n][:, None] for n in ("q", "k", "v")}
        out, state = _exact_forward(dict(case, T=1), dict(st, lens=None, **one))
        return out[:, 0], state
    return (_exact_forward if case["op"] == "forward" else _exact_backward)(case, st)


def _alive(case, st, t):
    if st["lens"] is None:
        return None
    return (st["lens"] > t)[:, None, None, None]


def _token(x, t, Hkv, alive):
    y = x[:, t].double()
    y = y.view(y.shape[0], Hkv, -1, y.shape[-1])                     # [B, Hkv, heads, d]
    return y if alive is None else torch.where(alive, y, torch.zeros_like(y))


def _exact_forward(case, st):
    Hkv, d, T = case["Hkv"], case["d"], case["T"]
    lam = torch.exp(st["log_decay"].double())[None, :, None, None]
    S = st["state"].double()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for t in range(T):
        al = _alive(case, st, t)
        q, k, v = (_token(st[n], t, Hkv, al) for n in ("q", "k", "v"))
        new = lam * S + k.transpose(-1, -2) * v
        S = new if al is None else torch.where(al, new, S)
        out[:, t] = (q @ S).reshape(out[:, t].shape) / math.sqrt(d)
    return out, S


def _exact_backward(case, st):
    Hkv, d, T = case["Hkv"], case["d"], case["T"]
    lam = torch.exp(st["log_decay"].double())[None, :, None, None]
    scale = 1.0 / math.sqrt(d)
    dq, dk, dv = (torch.zeros(st[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "v"))
    S = st["state"].double()
    for t in range(T):
        al = _alive(case, st, t)
        k, v, do = (_token(st[n], t, Hkv, al) for n in ("k", "v", "d_out"))
        new = lam * S + k.transpose(-1, -2) * v
        S = new if al is None else torch.where(al, new, S)
        dq[:, t] = (scale * (do @ S.transpose(-1, -2))).reshape(dq[:, t].shape)
    R = st["d_state"].double()                                       # dL/dS_t, from the last token to the first
    for t in reversed(range(T)):
        al = _alive(case, st, t)
        q, k, v, do = (_token(st[n], t, Hkv, al) for n in ("q", "k", "v", "d_out"))
        R = R + scale * (q.transpose(-1, -2) @ do)
        dk[:, t] = (v @ R.transpose(-1, -2)).reshape(dk[:, t].shape)
        dv[:, t] = (k @ R).reshape(dv[:, t].shape)
        R = lam * R if al is None else torch.where(al, lam * R, R)
    return dq, dk, dv, R


def _exact_rotation(case, st):
    rot, d = case["rot"], case["d"]
    half = rot // 2
    if case["pairs"] == "neighbours":
        first = torch.arange(0, rot, 2, device="cuda")
        second = first + 1
    else:
        first = torch.arange(half, device="cuda")
        second = first + half
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["positions"].double()[:, None] * st["freq"])[:, None]
    back = case["op"] == "rotate_backward"
    res_x, res_w = [], []
    for n in ("q", "k"):
        x, w = st[n].double(), st["w_" + n].double()
        norm = (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()
        y = (st["d_" + n].double() if back else x / norm * w).clone()
        turned = torch.complex(y[..., first], y[..., second]) * (z.conj() if back else z)
        y[..., first], y[..., second] = turned.real, turned.imag
        if not back:
            res_x.append(y)
            continue
        res_w.append((y * x / norm).sum((0, 1)))
        h = y * w
        res_x.append(h / norm - x * (h * x).sum(-1, keepdim=True) / (d * norm.pow(3)))
    return (*res_x, *res_w)
