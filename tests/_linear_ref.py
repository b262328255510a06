"""Linear attention with a decay for each head, and the norm and rotation of queries and keys, written out in 64
bits: token by token, as the formulas stand.  Shares no code with the library."""
import torch


def f64(x):
    return None if x is None else x.detach().double()


def linear_forward(q, k, v, log_decay, state=None, lens=None, scale=None):
    """q [B, T, Hq, d], k, v [B, T, Hkv, d] -> (out, state), float64."""
    q, k, v, g = f64(q), f64(k), f64(v), f64(log_decay)
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    scale = d ** -0.5 if scale is None else scale
    S = torch.zeros((B, Hkv, d, d), dtype=torch.float64, device=q.device) if state is None else f64(state).clone()
    lam = torch.exp(g)[None, :, None, None]
    out = torch.zeros_like(q)
    n = [T] * B if lens is None else [min(max(int(x), 0), T) for x in lens]
    for t in range(T):
        on = torch.tensor([t < x for x in n], device=q.device)
        if not bool(on.any()):
            break
        new = lam * S[on] + torch.einsum("bhi,bhj->bhij", k[on, t], v[on, t])
        S[on] = new
        out[on, t] = scale * torch.einsum("bhgi,bhij->bhgj", q[on, t].reshape(-1, Hkv, G, d), new).reshape(-1, Hq, d)
    return out, S


def linear_backward(d_out, q, k, v, log_decay, state=None, d_state=None, lens=None, scale=None):
    """Automatic differentiation of the token loop above, float64 -> (d_q, d_k, d_v, d_state_in)."""
    B, T, Hq, d = q.shape
    Hkv = k.shape[2]
    z = torch.zeros((B, Hkv, d, d), dtype=torch.float64, device=q.device)
    leaves = [f64(x).clone().requires_grad_() for x in (q, k, v)] + [(z if state is None else f64(state)).clone().requires_grad_()]
    n = [T] * B if lens is None else [min(max(int(x), 0), T) for x in lens]
    scale = d ** -0.5 if scale is None else scale
    lam = torch.exp(f64(log_decay))[:, None, None]
    loss = torch.zeros((), dtype=torch.float64, device=q.device)
    for b in range(B):
        S = leaves[3][b]
        for t in range(n[b]):
            S = lam * S + leaves[1][b, t][:, :, None] * leaves[2][b, t][:, None, :]
            o = scale * torch.einsum("hgi,hij->hgj", leaves[0][b, t].reshape(Hkv, -1, d), S).reshape(Hq, d)
            loss = loss + (o * f64(d_out)[b, t]).sum()
        if d_state is not None:
            loss = loss + (S * f64(d_state)[b]).sum()
    grads = torch.autograd.grad(loss, leaves, allow_unused=True)
    return tuple(torch.zeros_like(x) if g is None else g for x, g in zip(leaves, grads))


def rotate(y, positions, freq, interleaved, sign=1.0):
    """y [..., H, d] float64: its first 2 len(freq) features turned by positions * freq."""
    if freq is None or freq.numel() == 0:
        return y
    half = freq.numel()
    ang = f64(positions)[..., None, None] * f64(freq)
    c, s = torch.cos(ang), sign * torch.sin(ang)
    out = y.clone()
    ia = torch.arange(half, device=y.device) * 2 if interleaved else torch.arange(half, device=y.device)
    ib = ia + 1 if interleaved else ia + half
    out[..., ia] = y[..., ia] * c - y[..., ib] * s
    out[..., ib] = y[..., ia] * s + y[..., ib] * c
    return out


def norm_rotate(x, w, positions, freq, eps, interleaved):
    x = x if x.dtype == torch.float64 else f64(x)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * (w if w.dtype == torch.float64 else f64(w))
    return rotate(y, positions, freq, interleaved)
