"""Plain 64-bit implementations of the chunk and window operators, and the error bounds that the kernels' roundings allow."""
import math

import torch


class Seq:
    """What one (layer, sequence) of a cache holds: per KV head its keys, values, features and positions."""

    def __init__(self, Hkv, D, F):
        self.k = [torch.zeros((0, D), dtype=torch.bfloat16, device="cuda") for _ in range(Hkv)]
        self.v = [torch.zeros((0, D), dtype=torch.bfloat16, device="cuda") for _ in range(Hkv)]
        self.f = [torch.zeros((0, F), dtype=torch.float32, device="cuda") for _ in range(Hkv)]
        self.pos = [torch.zeros((0,), dtype=torch.int32, device="cuda") for _ in range(Hkv)]

    def __len__(self):
        return self.k[0].shape[0]

    def extend(self, k, v, pos=None, keep=None):
        """k, v [T][Hkv][D]; pos [T] or None (after the last pair that stays)."""
        for h in range(len(self.k)):
            n = len(self) if keep is None else keep
            if h > 0 and keep is None:
                n = self.k[h].shape[0]
            p = pos
            if p is None:
                first = int(self.pos[h][n - 1]) + 1 if n else 0
                p = torch.arange(first, first + k.shape[0], dtype=torch.int32, device="cuda")
            self.k[h] = torch.cat([self.k[h][:n], k[:, h]])
            self.v[h] = torch.cat([self.v[h][:n], v[:, h]])
            self.f[h] = torch.cat([self.f[h][:n], self.f[h].new_zeros((k.shape[0], self.f[h].shape[1]))])
            self.pos[h] = torch.cat([self.pos[h][:n], p])


def seen(pos, own_slot, own_pos, window, sinks):
    """[rows][n]: the pairs that queries with these slots and positions see."""
    at = torch.arange(pos.shape[0], device=pos.device)
    ok = at[None, :] <= own_slot[:, None]
    if window:
        x = pos.long()
        ok = ok & (x[None, :] <= own_pos.long()[:, None])
        ok = ok & ((own_pos.long()[:, None] - x[None, :] < window) | (x[None, :] < sinks))
    return ok


def attend(q, k, v, ok, scale):
    """q [rows][D], k, v [n][D] bf16, ok [rows][n]: out, log-sum-exp, probabilities and the bounds of out and lse.

    The bound of out: the result is rounded to bf16 once (half a step, 2^-8 relative), and so is every probability before
    it is multiplied with v (2^-8 of sum p |v|).  A score is a dot product of D terms accumulated in fp32: D 2^-23 of the
    sum of its terms' magnitudes (one truncation per addition), which moves a probability by as much, and the normalising
    sum by as much again; 2^-20 covers the exponentials, the running sums and the division.
    """
    rows, n, D = q.shape[0], k.shape[0], q.shape[1]
    if n == 0:
        z = torch.zeros((rows, D), dtype=torch.float64, device=q.device)
        empty = torch.full((rows,), -math.inf, dtype=torch.float64, device=q.device)
        return z, empty, z.new_zeros((rows, 0)), z + 1e-30, torch.zeros_like(empty) + 1e-6
    z = (q.double() @ k.double().T) * scale
    mag = (q.double().abs() @ k.double().abs().T) * scale
    z = torch.where(ok, z, torch.full_like(z, -math.inf))
    err = torch.where(ok, mag, torch.zeros_like(mag)).amax(1) * D * 2.0 ** -23 + 2.0 ** -20
    lse = torch.logsumexp(z, 1)
    p = torch.where(ok, torch.exp(z - lse[:, None]), torch.zeros_like(z))
    vv = torch.where(ok.any(0)[:, None], v.double(), torch.zeros_like(v, dtype=torch.float64))
    out = p @ vv
    spread = p @ vv.abs()
    tol = 2.0 ** -8 * (out.abs() + 1.01 * spread) + 2 * err[:, None] * spread + 1e-30
    return out, lse, p, tol, err + 2.0 ** -21 * lse.abs().nan_to_num(posinf=0.0)


def features(old, p, T):
    """Feature rows of one query head of every pair: old [n][6], p [T][n] probabilities of the chunk's queries."""
    new = old.double().clone()
    for i, w in enumerate((8, 16, 32)):
        new[:, i] = p[-w:].sum(0) / w
    new[:, 3] = p.sum(0) / T
    new[:, 4] = old[:, 4].double() + new[:, 3]
    new[:, 5] = 0.9 * old[:, 5].double() + new[:, 3]
    return new
