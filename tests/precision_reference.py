"""Caches and queries whose errors add up instead of averaging out, and what skvq_paged_weights may be off by on them (CPU, 64 bits).

Bounds count the steps of the kernels, not the sizes of random sums.  A tensor-core product adds 16 exact products and its accumulator after
aligning them to the largest and cutting each at 2^-25 of it (CUT allows 2^-23); an fp16 operand below 2^-14 is aligned as if it were 2^-14."""
import math

import torch

CUT = 2.0 ** -23
FINE = 2.0 ** -25
TAIL = 2.0 ** -16
EXP = 2.0 ** -22 + 2.0 ** -24      # of a probability: the exponential, its argument's product with log2(e) for arguments down to -1


def rounded_one_way(n, D, G, size, g, at_least=0.3):
    """Rows whose keys h c + z are positive and all lie above the nearest fp16 number by `at_least` of its steps or more:
    (codes uint8 [n, D], meta fp16 [n, D / G, 2])."""
    codes, meta = torch.zeros(n, D, dtype=torch.uint8), torch.zeros(n, D // G, 2, dtype=torch.float16)
    for t in range(n):
        for group in range(D // G):
            while True:
                h, z = ((torch.rand(2, generator=g) + 0.5) * torch.tensor([0.2, 1.0]) * size).half()
                x = h.double() * torch.arange(16) + z.double()
                step = torch.exp2(torch.floor(torch.log2(x)) - 10)
                good = torch.nonzero((x - x.half().double()) / step >= at_least)[:, 0]
                if len(good):
                    break
            pick = good[torch.randint(0, len(good), (G,), generator=g)]
            codes[t, group * G:(group + 1) * G] = pick.to(torch.uint8)
            meta[t, group, 0], meta[t, group, 1] = h, z
    return codes, meta


def keys(codes, meta):
    G = codes.shape[-1] // meta.shape[-2]
    m = meta.double()
    return (codes.double().unflatten(-1, (-1, G)) * m[..., :1] + m[..., 1:]).flatten(-2)


def two_parts(x):
    """A key as the sum of two fp16 numbers."""
    high = x.float().half()
    return high.double() + (x.float() - high.float()).half().double()


def queries_with_tails(rows, D, g):
    """fp16 [rows, D], all positive: every eighth is 1, the others lie between 2^-6 and 2^-5 with all eleven bits in use, the last one set:
    multiples of TAIL."""
    tails = (torch.randint(512, 1024, (rows, D), generator=g) * 2 + 1).double() * TAIL
    tails[:, ::8] = 1.0
    assert torch.equal(tails.half().double(), tails)
    return tails.half()


def cut_products(codes, meta, q, unit):
    """Scores [rows, n] whose products q c are cut to multiples of `unit`."""
    G = codes.shape[-1] // meta.shape[-2]
    c, x, m = codes.double().unflatten(-1, (-1, G)), q.double().unflatten(-1, (-1, G)), meta.double()
    a = (torch.floor(c[None] * x[:, None] / unit) * unit).sum(-1)      # [rows, n, groups]
    return (a * m[..., 0]).sum(-1) + torch.einsum("rg,ng->rn", x.sum(-1), m[..., 1])


def few_error(codes, meta, q, step=None):
    """Allowed error [rows, n] of q . K~ in the kernel for up to 16 rows: the sum over groups of h (q . c), and the sum of z (sum q) as one product
    of {h, z} words with {0, sum q} in two fp16 parts (2^-22 together).  Codes enter as c 2^-22 with q and as 16 c 2^-22 with q / 16: below
    2^-14, so aligned as if a code were 256 (16 where it takes the larger place, which shares products with the others).  `step`: q is a multiple of it."""
    D, G = codes.shape[-1], codes.shape[-1] // meta.shape[-2]
    c, x, m = codes.double().unflatten(-1, (-1, G)), q.double().unflatten(-1, (-1, G)), meta.double().abs()
    a = torch.einsum("ngj,rgj->rng", c, x.abs())
    top = torch.exp2(torch.floor(torch.log2(q.double().abs().amax(-1))))
    if step is not None:      # products are multiples of it, nothing is cut above it, and every partial sum has 24 bits
        products = c[None] * x[:, None] / step
        assert torch.equal(products, products.round()) and (256 * top * FINE <= step).all() and (a < 2.0 ** 24 * step).all()
        code_error = torch.zeros_like(a)
    else:
        code_error = G / 16 * 17 * CUT * torch.maximum(256 * top[:, None, None], a)
    z = torch.einsum("rg,ng->rn", x.sum(-1).abs(), m[..., 1])
    ops = (D // G + 3) * 2.0 ** -24 * ((a * m[..., 0]).sum(-1) + z)
    return (code_error * m[..., 0]).sum(-1) + z * (17 * CUT + 2.0 ** -22) + ops


def many_error(codes, meta, q):
    """Allowed error [rows, n] of q . K~ in the kernel for more rows: a key as two fp16 parts (2^-22 of it), D / 16 products of the low parts,
    then D / 16 of the high ones on top."""
    D = codes.shape[-1]
    K, x = keys(codes, meta).abs(), q.double().abs()
    s = x @ K.t()
    least = 2.0 ** -14 * x.amax(-1, keepdim=True)      # what an operand below 2^-14 is aligned as
    return 2.0 ** -22 * s + D / 16 * 17 * CUT * (torch.maximum(s, least) + torch.maximum(s * 2.0 ** -11, least)) + 2.0 ** -24 * s


def weights(scores, errors, lse, sm_scale):
    """(weights [n], allowed error [n]) of scores [rows, n] before the scale."""
    e = sm_scale * scores - lse.double()[:, None]
    p = torch.exp(e)
    # the scale as fp32; the difference to lse is rounded once
    off = sm_scale * errors + (sm_scale * scores).abs() * 2.0 ** -24 + e.abs() * (2.0 ** -23 + 2.0 ** -24)
    rows = scores.shape[0]
    return p.sum(0), (p * (torch.expm1(off) + EXP)).sum(0) + p.sum(0) * (rows + 2) * CUT + rows * 2.0 ** -120


def scale_for(scores, top):
    """An exact scale that brings the largest score to about `top`."""
    return 2.0 ** math.floor(math.log2(top / float(scores.abs().max())))
