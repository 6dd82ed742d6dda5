"""Rotations with several axes, accumulated attention weights and eviction, written plainly (64 bits where there are numbers; CPU, no
library code)."""
import math

import torch

import paged_reference as ref


def axis_angles(table, positions, of_pair):
    """[T, pairs, 2]: pair j of token t from row positions[of_pair[j], t]."""
    return torch.stack([table[positions[a].long(), j] for j, a in enumerate(of_pair)], 1)


def weights(r, b, q, lse, old, sm_scale, causal=True, last=0, length=None):
    """What skvq_paged_weights gives sequence b of a paged_reference.Reference: (float64 [H, L], allowed error [H, L]).

    The error counts, for every row: a score's sum of D terms q (h code), each held as code + 8 steps at most, and NG terms q z, in fp32
    with truncating adders (2^-23 a term; the parts of a group's sum are formed apart); the score's and the lse's products with
    the scale (2^-22 of each); an exponential good to 2^-22; then fp32 sums."""
    n, L = q.shape[0], len(r.rows[b])
    if r.rot_dim and n:
        pos = torch.arange(L - n, L)
        turned = ref.rotate32(q, r.table[pos.clamp(min=0)], r.rot_dim, r.interleaved)
        q = torch.where((pos >= 0)[:, None, None], turned, q)
    K = r.values(b, "k")
    size = torch.zeros(L, r.H, r.D, dtype=torch.float64)
    for t, row in enumerate(r.rows[b]):
        if t >= L - r.W:
            size[t] = row[0].double().abs()
        else:
            m = row[3].double()
            size[t] = ((row[2].double().unflatten(-1, (-1, r.G)) + 8) * m[..., :1].abs() + m[..., 1:].abs()).flatten(-2)
    out, err = torch.zeros(r.H, L, dtype=torch.float64), torch.zeros(r.H, L, dtype=torch.float64)
    fresh = max(L - n, 0)
    if old is not None:
        out[:, :fresh] = old[:, :fresh].double()
    rep, first = r.Hq // r.H, max(n - last, 0) if last else 0
    for h in range(r.H):
        rows = 0
        for i in range(first, n):
            lim = max(0, L - n + i + 1) if causal else L
            for hq in range(h * rep, (h + 1) * rep):
                qr = q[i, hq].double()[r.rk[h]]
                if not math.isfinite(float(lse[i, hq])) or not torch.isfinite(qr).all() or lim == 0:
                    continue
                rows += 1
                s = sm_scale * (K[:lim, h] @ qr)
                p = torch.exp(s - float(lse[i, hq]))
                ds = abs(sm_scale) * (size[:lim, h] @ qr.abs()) * (r.D + 8) * 2.0 ** -23
                out[h, :lim] += p
                err[h, :lim] += p * torch.expm1(ds + (s.abs() + abs(float(lse[i, hq]))) * 2.0 ** -22 + 2.0 ** -22)
        err[h] += out[h].abs() * (rows + 2) * 2.0 ** -23 + rows * 2.0 ** -120
    return out, err


def chosen(w, L, keep, first, recent):
    """The kept tokens of one head, in order."""
    if L <= keep:
        return list(range(L))
    middle = [(-math.inf if math.isnan(float(x)) else float(x), math.isnan(float(x)), t) for t, x in zip(range(first, L - recent), w[first:L - recent])]
    middle.sort(key=lambda e: (e[1], -e[0], e[2]))      # numbers first, the largest first, the lower token first
    best = sorted(e[2] for e in middle[:keep - first - recent])
    return list(range(first)) + best + list(range(L - recent, L))
