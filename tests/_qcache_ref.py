"""The 8-bit cache written out in 64 bits, unit by unit, as its formulas stand.  Shares no code with the library."""
import math

import numpy as np
import torch

BLOCK = 32
NAMES = ("k", "v", "k_scale", "v_scale", "weight", "position", "state")


class Ref:
    """The planes of a cache as numpy arrays; its methods change them as the calls do."""

    def __init__(self, planes):
        for name, t in zip(NAMES, planes):
            setattr(self, name, t.detach().cpu().numpy().copy())
        self.B, self.H, self.C, self.d = self.k.shape

    def values(self, p, b, h, n):
        codes, scale = getattr(self, p)[b, h, :n], getattr(self, p + "_scale")[b, h]
        return codes.astype(np.float64) * scale[np.arange(n) // BLOCK].astype(np.float64)[:, None]

    def _write(self, p, b, h, slots, x, end):
        """Rows x into `slots`, where no slot from `end` on holds anything."""
        codes, scale = getattr(self, p)[b, h], getattr(self, p + "_scale")[b, h]
        slots = np.asarray(slots, dtype=np.int64)                     # ascending
        assert (np.diff(slots) > 0).all()
        for blk in np.unique(slots // BLOCK).tolist():
            mine = slice(*np.searchsorted(slots, [blk * BLOCK, (blk + 1) * BLOCK]).tolist())
            rows = slots[mine].tolist()
            stay = [j for j in range(blk * BLOCK, min(blk * BLOCK + BLOCK, end)) if j not in rows]
            new = x[mine]
            s = float(scale[blk])
            if not np.isfinite(new).all() or (stay and s != s):
                scale[blk] = np.nan
                codes[rows] = 0
                continue
            amax = float(np.abs(new).max())
            if not stay or s == 0:
                s = float(np.float32(max(amax / 127, 2.0 ** -126))) if amax > 0 else 0.0
            else:
                old = s
                while amax > 127.5 * s:
                    s *= 2
                codes[stay] = np.rint(codes[stay] * (old / s)).astype(np.int8)
            scale[blk] = s
            codes[rows] = np.clip(np.rint(new / s), -127, 127).astype(np.int8) if s else 0

    def append(self, k, v, lens=None):
        T = k.shape[1]
        x = {"k": k.double().cpu().numpy(), "v": v.double().cpu().numpy()}
        for b in range(self.B):
            held, seen = int(self.state[0, b]), int(self.state[1, b])
            n = min(T if lens is None else min(max(int(lens[b]), 0), T), self.C - held)
            slots = np.arange(held, held + n)
            for h in range(self.H):
                for p in "kv":
                    self._write(p, b, h, slots, x[p][b, :n, h], held)
                self.weight[b, h, slots] = 0
                self.position[b, h, slots] = seen + np.arange(n)
            self.state[0, b], self.state[1, b] = held + n, seen + n

    def evict(self, keep, recent=0):
        for b in range(self.B):
            held, seen = int(self.state[0, b]), int(self.state[1, b])
            if held <= keep:
                continue
            for h in range(self.H):
                w, pos = self.weight[b, h, :held], self.position[b, h, :held]
                order = sorted((j for j in range(held) if pos[j] < seen - recent),
                               key=lambda j: (w[j] != w[j], float(w[j]) if w[j] == w[j] else 0.0, j))
                gone = set(order[:held - keep])
                assert len(gone) == held - keep
                dest = np.array([j for j in range(keep) if j in gone], dtype=np.int64)
                src = np.array([j for j in range(keep, held) if j not in gone], dtype=np.int64)
                assert len(dest) == len(src)
                if len(dest) == 0:
                    continue
                for p in "kv":
                    self._write(p, b, h, dest, self.values(p, b, h, held)[src], keep)
                self.weight[b, h, dest] = self.weight[b, h, src]
                self.position[b, h, dest] = self.position[b, h, src]
            self.state[0, b] = keep

    def attend(self, q, lens=None, scale=None, cap=0.0, device="cpu"):
        """-> (out, added weight, sum_j p_j |v_j| for each output, largest sum_i |q_i k_i| scale, largest |v|), float64."""
        B, T, Hq, d = q.shape
        G = Hq // self.H
        scale = 1 / math.sqrt(d) if scale is None else scale
        out, mag = torch.zeros((B, T, Hq, d), dtype=torch.float64), torch.zeros((B, T, Hq, d), dtype=torch.float64)
        added = torch.zeros((B, self.H, self.C), dtype=torch.float64)
        big = loudest = 0.0
        for b in range(B):
            held = int(self.state[0, b])
            n = T if lens is None else min(max(int(lens[b]), 0), T)
            if n == 0 or held == 0:
                continue
            sees = torch.clamp(held - n + 1 + torch.arange(n, device=device), min=0)
            hidden = torch.arange(held, device=device)[None, :] >= sees[:, None]
            for h in range(self.H):
                K, V = (torch.from_numpy(self.values(p, b, h, held)).to(device) for p in "kv")
                x = q[b, :n, h * G:(h + 1) * G].double().to(device).transpose(0, 1)          # [G, n, d]
                s = x @ K.T * scale
                big = max(big, float((x.abs() @ K.abs().T).max()) * scale)
                loudest = max(loudest, float(V.abs().max()))
                if cap:
                    s = cap * torch.tanh(s / cap)
                s = s.masked_fill(hidden, -math.inf)
                m = s.amax(-1, keepdim=True)
                p = torch.exp(s - torch.where(torch.isinf(m), 0.0, m))
                total = p.sum(-1, keepdim=True)
                p = p / torch.where(total == 0, 1.0, total)
                out[b, :n, h * G:(h + 1) * G] = (p @ V).transpose(0, 1).cpu()
                mag[b, :n, h * G:(h + 1) * G] = (p @ V.abs()).transpose(0, 1).cpu()
                added[b, h, :held] = p.sum((0, 1)).cpu()
        return out, added, mag, big, loudest
