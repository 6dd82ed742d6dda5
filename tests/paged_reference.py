"""Rotation, paged cache and attention over it, written plainly in 64 bits on the CPU (torch tensors; no library code).

Rounded steps that are part of the definitions -- rotated keys and queries held in the tensors' type, fp16 parameters -- are
rounded here too; everything else is exact to 64 bits."""
import math

import torch


def table64(rot_dim, n, base=10000.0):
    f = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    a = torch.arange(n, dtype=torch.float64)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1)


def rotate(x, cs, rot_dim, interleaved, inverse=False):
    """x [T, H, D], cs [T, rot_dim/2, 2] -> float64 [T, H, D]."""
    y = x.double().clone()
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double()
    if inverse:
        s = -s
    first, second = (slice(0, rot_dim, 2), slice(1, rot_dim, 2)) if interleaved else (slice(0, rot_dim // 2), slice(rot_dim // 2, rot_dim))
    x1, x2 = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def rotate32(x, cs, rot_dim, interleaved, inverse=False):
    """The documented rounding: products and their sum in fp32, then the type."""
    y = x.clone()
    c, s = cs[:, None, :, 0].float(), cs[:, None, :, 1].float()
    if inverse:
        s = -s
    first, second = (slice(0, rot_dim, 2), slice(1, rot_dim, 2)) if interleaved else (slice(0, rot_dim // 2), slice(rot_dim // 2, rot_dim))
    x1, x2 = x[..., first].float(), x[..., second].float()
    a, b, d, e = x1 * c, x2 * s, x2 * c, x1 * s
    y[..., first], y[..., second] = (a - b).to(x.dtype), (d + e).to(x.dtype)
    return y


def quantize(xr, alpha, G):
    """xr [..., D] (stored order) -> codes uint8 [..., D], meta fp16 [..., D/G, 2]; fp32 as documented."""
    x = xr.float().unflatten(-1, (-1, G))
    lo, hi = alpha * x.amin(-1) + 0.0, alpha * x.amax(-1) + 0.0
    meta = torch.stack(((hi - lo) * torch.tensor(1.0 / 15.0, dtype=torch.float32), lo), -1).half()
    h, z = meta[..., :1].float(), meta[..., 1:].float()
    c = torch.where(h != 0, torch.round((x - z) / h).clamp(0, 15), torch.zeros_like(x))
    return c.to(torch.uint8).flatten(-2), meta


class Reference:
    """The cache of every sequence as plain rows: tokens in order, stored channel order."""

    def __init__(self, n_seqs, Hq, H, D, G, W, dtype, reorder_k=None, reorder_v=None, alpha_k=None, alpha_v=None, table=None,
                 rot_dim=0, interleaved=False):
        self.Hq, self.H, self.D, self.G, self.W, self.dtype = Hq, H, D, G, W, dtype
        ident = torch.arange(D).repeat(H, 1)
        self.rk = ident if reorder_k is None else reorder_k.long()
        self.rv = ident if reorder_v is None else reorder_v.long()
        one = torch.ones(H, D // G)
        self.ak, self.av = (one if alpha_k is None else alpha_k), (one if alpha_v is None else alpha_v)
        self.table, self.rot_dim, self.interleaved = table, rot_dim, interleaved
        self.rows = [[] for _ in range(n_seqs)]      # per token: (k fp, v fp, k codes, k meta, v codes, v meta), stored order

    def append(self, b, k, v):
        """k, v [n, H, D] in the type, source order."""
        n, t0 = k.shape[0], len(self.rows[b])
        if self.rot_dim and n:
            k = rotate32(k, self.table[t0:t0 + n], self.rot_dim, self.interleaved)
        kr = torch.stack([k[:, h][:, self.rk[h]] for h in range(self.H)], 1)
        vr = torch.stack([v[:, h][:, self.rv[h]] for h in range(self.H)], 1)
        (kc, km), (vc, vm) = quantize(kr, self.ak, self.G), quantize(vr, self.av, self.G)
        self.rows[b] += [(kr[i], vr[i], kc[i], km[i], vc[i], vm[i]) for i in range(n)]

    def truncate(self, b, length):
        self.rows[b] = self.rows[b][:length]

    def values(self, b, which, window=True):
        """float64 [L, H, D] in stored order: h code + z, the newest W tokens unquantized."""
        L = len(self.rows[b])
        out = torch.zeros(L, self.H, self.D, dtype=torch.float64)
        for t, row in enumerate(self.rows[b]):
            if window and t >= L - self.W:
                out[t] = row[0 if which == "k" else 1].double()
            else:
                c, m = (row[2], row[3]) if which == "k" else (row[4], row[5])
                m = m.double()
                out[t] = (c.double().unflatten(-1, (-1, self.G)) * m[..., :1] + m[..., 1:]).flatten(-2)
        return out

    def score_error(self, b):
        """float64 [L, H, D]: bound of a score's error per unit of |q'_j|.  The sum of D terms h code + |z| (|k| in the window) in
        truncating fp32 (2^-23 each), keys formed in fp16 (2^-11, in the kernel for many rows); codes that enter the product as
        1024 + c: 16 additions truncated at 2^-23 of sums of 1024 |q'| h."""
        L = len(self.rows[b])
        out = torch.zeros(L, self.H, self.D, dtype=torch.float64)
        for t, row in enumerate(self.rows[b]):
            if t >= L - self.W:
                out[t] = row[0].double().abs() * (self.D * 2.0 ** -23 + 2.0 ** -11)
            else:
                m = row[3].double()
                h = m[..., :1]
                mag = row[2].double().unflatten(-1, (-1, self.G)) * h + m[..., 1:].abs()
                out[t] = (mag * (self.D * 2.0 ** -23 + 2.0 ** -11) + h * (16 * 1024 * 2.0 ** -23)).flatten(-2)
        return out

    def attention(self, b, q, sm_scale, causal=True, length=None):
        """q [n, Hq, D] -> (out float64 [n, Hq, D] in source order, lse [n, Hq], allowed error [n, Hq, D], of lse [n, Hq]).

        The error bound counts: the scores' (score_error), probabilities and values rounded to fp16 (2^-11 each), fp32 sums of L
        probabilities with truncating adders, ex2 to 2^-22."""
        n, L = q.shape[0], len(self.rows[b])
        if self.rot_dim and n:
            pos = torch.arange(L - n, L)
            turned = rotate32(q, self.table[pos.clamp(min=0)], self.rot_dim, self.interleaved)
            q = torch.where((pos >= 0)[:, None, None], turned, q)
        K, V, off = self.values(b, "k"), self.values(b, "v"), self.score_error(b)
        out = torch.zeros(n, self.Hq, self.D, dtype=torch.float64)
        lse = torch.full((n, self.Hq), -math.inf, dtype=torch.float64)
        err, err_lse = torch.zeros_like(out), torch.zeros(n, self.Hq, dtype=torch.float64)
        rep = self.Hq // self.H
        half_step = torch.finfo(self.dtype).eps / 2
        for i in range(n):
            lim = max(0, L - n + i + 1) if causal else L
            if lim == 0:
                continue
            for hq in range(self.Hq):
                h = hq // rep
                qr = q[i, hq].double()[self.rk[h]]
                s = sm_scale * (K[:lim, h] @ qr)
                m = s.max()
                p = torch.exp(s - m)
                l = p.sum()
                p = p / l
                o = p @ V[:lim, h]
                a = p @ V[:lim, h].abs()
                ds = abs(sm_scale) * float((off[:lim, h] @ qr.abs()).max())
                # a probability far below the largest is held to 2^-39 of it (fp16 steps of 2^-24 under a factor 2^14, half of one)
                floor = float((V[:lim, h].abs().sum(0) / l).max()) * 2.0 ** -39
                out[i, hq, self.rv[h]] = o
                err[i, hq, self.rv[h]] = a * (2.0 ** -10 + 2 * ds + 2.0 ** -21 + lim * 2.0 ** -23) + o.abs() * half_step * 1.01 + floor + 1e-7
                lse[i, hq] = m + torch.log(l)
                err_lse[i, hq] = ds + 2.0 ** -21 + lim * 2.0 ** -23 + abs(float(lse[i, hq])) * 2.0 ** -22
        return out, lse, err, err_lse
