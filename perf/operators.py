"""Cases of the paged-cache operators: rotary positions, appending to a paged 4-bit cache, attention over it.

``own`` False: every operator in elementary torch operations, in 32 bits, rounded once at the end.  ``own`` True: the
calls a serving program makes of the library.  Shapes follow the benchmark workloads of this repository: 32 query heads
over 32 or 8 KV heads of 128 channels, contexts of 4096 to 131072 tokens, groups of 32, 64 and 128 channels, windows of 128
and 256 tokens, the ragged serving mix of 64 sequences with 1024 to 16384 tokens; keys with outlier channels.

A case's sequence lengths follow from its sizes alone (the seed makes the values), so that ``work`` is exact.

Definitions.  Rotation: y1 = x1 c - x2 s, y2 = x2 c + x1 s in fp32, the products rounded, then the sum, then to the
tensor's type.  Quantizer, per token and group of channels (reordered): lo = alpha min, hi = alpha max,
h = fp16((hi - lo) / 15), z = fp16(lo), code = clamp(rint((x - z) / h), 0, 15), 0 where h is 0; value h code + z.  Row of
codes: code j in bits [4 j, 4 j + 4).  The newest ``window`` tokens of a sequence are read unquantized from a ring (token t
in slot t mod ring), older ones from the pages.
"""
import math
import random

import torch

own = False

OUTLIERS, OUTLIER_SCALE, ALPHA = 4, 15.0, 0.95
DTYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------ cases
def rope(name, tokens, q_heads, kv_heads, head_dim, rot_dim, interleaved, inverse, dtype, context):
    return {"name": name, "op": "rope", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot_dim": rot_dim, "interleaved": interleaved, "inverse": inverse, "dtype": dtype, "context": context}


def paged(name, op, seqs, new, prior, heads, head_dim, group, window, page, rot_dim, interleaved, dtype, causal=True):
    return {"name": name, "op": op, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "prior_lo": prior[0], "prior_hi": prior[1],
            "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "group": group, "window": window, "page": page,
            "rot_dim": rot_dim, "interleaved": interleaved, "dtype": dtype, "causal": causal}


def listed():
    return [
        # one decode step of the ragged serving mix: queries and keys of 64 sequences, each at its own position
        rope("rope decode", 64, 32, 8, 128, 128, False, False, "bfloat16", 16384),
        # a prompt of 32k tokens, grouped-query shape
        rope("rope prompt", 32768, 32, 8, 128, 128, False, False, "float16", 32768),
        # gradients of a rotation of half the head in neighbouring pairs, an odd number of tokens
        rope("rope backward partial", 8191, 32, 32, 128, 64, True, True, "bfloat16", 16384),
        # one decode step of the serving mix: a token for each of 64 sequences
        paged("append decode", "append", 64, (1, 1), (1023, 16383), (32, 32), 128, 64, 256, 64, 128, False, "float16"),
        # a whole 32k prompt of the multi-head shape at once
        paged("append prompt", "append", 1, (32768, 32768), (0, 0), (32, 32), 128, 128, 128, 64, 128, False, "float16"),
        # a mixed step: decode tokens beside ragged prompt chunks, narrow heads, half of each rotated in neighbouring pairs
        paged("append mixed", "append", 17, (1, 2047), (0, 4095), (32, 8), 64, 32, 128, 16, 32, True, "bfloat16"),
        # the smallest context of the benchmark: one query over 4096 tokens, where latency counts
        paged("attention short", "attention", 1, (1, 1), (4095, 4095), (32, 32), 128, 128, 128, 64, 128, False, "float16"),
        # a decode step of the serving mix
        paged("attention serving", "attention", 64, (1, 1), (1023, 16383), (32, 32), 128, 64, 256, 64, 128, False, "float16"),
        # a decode step over long contexts, grouped-query shape with fine groups
        paged("attention long", "attention", 4, (1, 1), (131071, 131071), (32, 8), 128, 32, 128, 64, 128, False, "bfloat16"),
        # four drafted tokens for each of 16 sequences, verified in one pass
        paged("attention drafts", "attention", 16, (4, 4), (1020, 16380), (32, 8), 128, 64, 256, 32, 128, False, "bfloat16"),
        # a chunk of a long prompt: 2048 queries over 32k tokens
        paged("attention chunk", "attention", 1, (2048, 2048), (30720, 30720), (32, 8), 128, 64, 256, 64, 128, False, "float16"),
        # ragged prompts from their first token, narrow heads
        paged("attention prompts", "attention", 9, (1, 4095), (0, 0), (32, 32), 64, 32, 128, 16, 64, False, "bfloat16"),
    ]


def log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = {"bytes": 1.3e9, "flops": 1.0e12, "scores": 1.6e9, "values": 3.0e9}
    while True:
        op = rng.choice(["rope", "append", "attention", "attention"])
        dtype = rng.choice(sorted(DTYPES))
        head_dim = rng.choice([64, 128, 128])
        rot_dim = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
        inter = rng.random() < 0.5
        q_heads, kv_heads = rng.choice([(32, 32), (32, 8), (32, 16), (32, 4), (8, 8), (24, 8)])
        if op == "rope":
            c = rope("", log_int(rng, 1, 32768), q_heads, kv_heads, head_dim, rot_dim, inter, rng.random() < 0.4, dtype, 32768)
        else:
            seqs = log_int(rng, 1, 64)
            if op == "append":
                hi = rng.choice([1, log_int(rng, 2, 16384)])
            else:
                hi = rng.choice([1, 1, log_int(rng, 2, 16), log_int(rng, 17, 4096)])
            prior = log_int(rng, 1, 131072)
            prior = (0, 0) if hi > 1 and rng.random() < 0.3 else (prior // rng.choice([1, 2, 8]), prior)
            group = rng.choice([g for g in (32, 64, 128) if g <= head_dim])
            c = paged("", op, seqs, (max(1, hi // rng.choice([1, 4, 64])), hi), prior, (q_heads, kv_heads), head_dim, group,
                      rng.choice([0, 128, 256]), rng.choice([16, 32, 64, 128]), rng.choice([0, rot_dim]), inter, dtype,
                      op == "append" or rng.random() < 0.8)
        del c["name"]
        w = work(c)
        values = scores = 0
        if op != "rope":
            new, total = lengths(c)
            values = len(total) * max(total) * kv_heads * head_dim
            scores = len(total) * max(new) * max(total) * q_heads if op == "attention" else 0
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and scores <= most["scores"] and values <= most["values"]:
            return c


def lengths(c):
    """New tokens and total length of every sequence: from the case's sizes alone."""
    r = random.Random("%d %d %d %d %d" % (c["seqs"], c["new_lo"], c["new_hi"], c["prior_lo"], c["prior_hi"]))
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["seqs"])]
    return new, [n + r.randint(c["prior_lo"], c["prior_hi"]) for n in new]


def work(case):
    c = case
    if c["op"] == "rope":
        n = c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["head_dim"]
        pairs = c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["rot_dim"] // 2
        return {"bytes": 2 * n * 2 + c["tokens"] * (4 * c["rot_dim"] + 4), "flops": 6 * pairs}
    new, total = lengths(c)
    T, H, D, W = sum(new), c["kv_heads"], c["head_dim"], c["window"]
    row = D // 2 + 4 * (D // c["group"])      # one token's codes and parameters, keys or values
    table = T * 4 * c["rot_dim"]
    if c["op"] == "append":
        ring = sum(min(n, W) for n in new) * H * D * 2
        # keys and values in, codes and ring out; then the new rows read back as values
        return {"bytes": 2 * (T * H * D * 2 + T * H * row + ring) + 2 * (T * H * row + T * H * D * 2) + table,
                "flops": 2 * T * H * D * 10}
    pairs = 0
    held = 0
    for n, L in zip(new, total):
        pairs += n * L - n * (n - 1) // 2 if c["causal"] else n * L
        held += 2 * H * (max(L - W, 0) * row + min(L, W) * D * 2)
    return {"bytes": held + 2 * T * c["q_heads"] * D * 2 + table, "flops": 4 * D * c["q_heads"] * pairs}


# ------------------------------------------------------------------------------------------------ inputs
def angles(n, rot_dim, device="cuda"):
    """cos and sin of position p times 10000 ** (-2 j / rot_dim): fp32 [n, rot_dim / 2, 2], computed in 64 bits."""
    f = 10000.0 ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    a = torch.arange(n, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack((a.cos(), a.sin()), -1).float()


def key_sigma(g, heads, dim):
    """Per-channel scale of the keys, a few outlier channels in every head."""
    s = torch.exp(0.5 * torch.randn(heads, dim, generator=g, device="cuda"))
    at = torch.rand(heads, dim, generator=g, device="cuda").argsort(1)[:, :OUTLIERS]
    return s.scatter(1, at, s.gather(1, at) * OUTLIER_SCALE)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t = DTYPES[c["dtype"]]
    D, H, Hq = c["head_dim"], c["kv_heads"], c["q_heads"]
    s = {"c": c}
    if c["op"] == "rope":
        T = c["tokens"]
        # queries, keys and values of a layer lie side by side, as one projection writes them
        qkv = torch.randn(T, Hq + 2 * H, D, generator=g, device="cuda").to(t)
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        if T <= 256:
            s["positions"] = torch.randint(0, c["context"], (T,), generator=g, device="cuda", dtype=torch.int32)
        else:
            s["positions"] = torch.arange(T, device="cuda", dtype=torch.int32) % c["context"]
        s["table"] = angles(c["context"], c["rot_dim"])
        if own:
            from paper_2405_06219_b200 import binding
            s["rope"] = binding.RopeTable(s["table"], c["rot_dim"], c["interleaved"])
        return s
    new, total = lengths(c)
    T, P, W = sum(new), c["page"], c["window"]
    pages = [-(-n // P) for n in total]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(c["seqs"], max(pages), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    sigma = key_sigma(g, H, D)
    s["reorder_k"] = sigma.argsort(1).to(torch.int32)
    s["reorder_v"] = torch.rand(H, D, generator=g, device="cuda").argsort(1).to(torch.int32)
    s["alpha"] = torch.full((H, D // c["group"]), ALPHA, device="cuda")
    s["page_table"] = table
    s["lens"] = torch.tensor(total, dtype=torch.int32, device="cuda")
    s["starts"] = torch.tensor([sum(new[:b]) for b in range(c["seqs"] + 1)], dtype=torch.int32, device="cuda")
    s["new"], s["total"] = new, total
    s["sm_scale"] = 1.0 / math.sqrt(D)
    s["table"] = angles(max(total), c["rot_dim"]) if c["rot_dim"] else None
    ng = D // c["group"]
    sigma_r = sigma.gather(1, s["reorder_k"].long())
    shape = (n_pages, H, P)
    s["k_codes"], s["v_codes"] = (torch.zeros(*shape, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
    s["k_meta"], s["v_meta"] = (torch.zeros(*shape, ng, 2, dtype=torch.float16, device="cuda") for _ in range(2))
    s["k_win"], s["v_win"] = (torch.zeros(c["seqs"], H, W, D, dtype=t, device="cuda") for _ in range(2))
    if c["op"] == "append":
        s["k"] = (torch.randn(T, H, D, generator=g, device="cuda") * sigma).to(t)
        s["v"] = torch.randn(T, H, D, generator=g, device="cuda").to(t)
    else:
        s["q"] = torch.randn(T, Hq, D, generator=g, device="cuda").to(t)
        step = max(1, (1 << 27) // (H * P * D))
        for lo in range(0, n_pages, step):
            n = min(step, n_pages - lo)
            for name, scale in (("k", sigma_r[None, :, None]), ("v", 1.0)):
                x = (torch.randn(n, H, P, D, generator=g, device="cuda") * scale).to(t).float()
                codes, meta = quantize(x, s["alpha"][None, :, None], c["group"])
                s[name + "_codes"][lo:lo + n] = codes[..., 0::2] | codes[..., 1::2] << 4
                s[name + "_meta"][lo:lo + n] = meta
        s["k_win"].copy_(torch.randn(s["k_win"].shape, generator=g, device="cuda") * sigma_r[None, :, None])
        s["v_win"].copy_(torch.randn(s["v_win"].shape, generator=g, device="cuda"))
    if own:
        from paper_2405_06219_b200 import binding
        s["cache"] = binding.SkvqPagedCache(
            Hq, H, D, c["group"], W, P, n_pages, c["seqs"], dtype=t, reorder_k=s["reorder_k"], reorder_v=s["reorder_v"],
            alpha_k=s["alpha"], alpha_v=s["alpha"],
            buffers={n: s[n] for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")})
        s["batch"] = s["cache"].batch(table, s["lens"], s["starts"], n_tokens=T, max_new=max(new), max_len=max(total))
        s["rope"] = binding.RopeTable(s["table"], c["rot_dim"], c["interleaved"]) if c["rot_dim"] else None
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def quantize(x, alpha, group):
    """fp32 x [..., D] -> codes uint8 [..., D] and fp16 parameters [..., D / group, 2] {h, z}."""
    xg = x.unflatten(-1, (-1, group))
    lo = alpha * xg.amin(-1) + 0.0
    hi = alpha * xg.amax(-1) + 0.0
    meta = torch.stack(((hi - lo) / 15.0, lo), -1).half()
    h, z = meta[..., 0:1].float(), meta[..., 1:2].float()
    codes = torch.where(h != 0, torch.round((xg - z) / h).clamp(0, 15), torch.zeros_like(xg))
    return codes.to(torch.uint8).flatten(-2), meta


def rotate(x, cs, rot_dim, interleaved, inverse=False):
    """x [T, H, D] in its type, cs fp32 [T, rot_dim / 2, 2] -> the rotated x in its type."""
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if inverse:
        s = -s
    r = x[..., :rot_dim].float()
    if interleaved:
        x1, x2 = r[..., 0::2], r[..., 1::2]
        y = torch.stack((x1 * c - x2 * s, x2 * c + x1 * s), -1).flatten(-2)
    else:
        x1, x2 = r[..., :rot_dim // 2], r[..., rot_dim // 2:]
        y = torch.cat((x1 * c - x2 * s, x2 * c + x1 * s), -1)
    return torch.cat((y.to(x.dtype), x[..., rot_dim:]), -1)


def token_rows(s):
    """Sequence and position of every row of the packed tokens."""
    n = s["starts"][1:] - s["starts"][:-1]
    T = sum(s["new"])
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), n, output_size=T)
    at = torch.arange(T, device="cuda") - s["starts"][seq]
    return seq, (s["lens"] - n)[seq] + at, at


def rotated(s, x, position):
    c = s["c"]
    return rotate(x, s["table"][position], c["rot_dim"], c["interleaved"]) if c["rot_dim"] else x


def plain_append(s):
    c = s["c"]
    T, H, D = s["k"].shape
    W = c["window"]
    seq, position, _ = token_rows(s)
    out = []
    for x, reorder, ring in ((rotated(s, s["k"], position), s["reorder_k"], s["k_win"]), (s["v"], s["reorder_v"], s["v_win"])):
        at = reorder.long().expand(T, H, D)
        xr = x.gather(2, at)
        codes, meta = quantize(xr.float(), s["alpha"], c["group"])
        value = codes.unflatten(-1, (-1, c["group"])).float() * meta[..., 0:1].float() + meta[..., 1:2].float()
        out.append(torch.empty(T, H, D, dtype=x.dtype, device="cuda").scatter_(2, at, value.flatten(-2).to(x.dtype)))
        if W:
            # the rows that stay in the window; the others are written to a slot that the last of them keeps
            last = position >= s["lens"][seq] - W
            rows = torch.nonzero(last, as_tuple=True)[0]
            ring[seq[rows], :, position[rows] % W] = xr[rows]
    return {"k": out[0], "v": out[1], "k_win": s["k_win"], "v_win": s["v_win"]}


def held_values(s, name):
    """The cache as fp32 [B, H, Lmax, D], reordered channels: pages, the window's tokens from the ring."""
    c = s["c"]
    W, P = c["window"], c["page"]
    codes = s[name + "_codes"][s["page_table"].long()].transpose(1, 2).flatten(2, 3)      # [B, H, L, D / 2]
    meta = s[name + "_meta"][s["page_table"].long()].transpose(1, 2).flatten(2, 3).float()
    x = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).unflatten(-1, (-1, c["group"])).float()
    x = (x.mul_(meta[..., 0:1]).add_(meta[..., 1:2])).flatten(-2)
    if W:
        t = s["lens"][:, None].long() - W + torch.arange(W, device="cuda")
        b = torch.arange(c["seqs"], device="cuda")[:, None].expand_as(t)
        b, t = b[t >= 0], t[t >= 0]
        x[b, :, t] = s[name + "_win"][b, :, t % W].float()
    return x


def plain_attention(s):
    c = s["c"]
    T, Hq, D = s["q"].shape
    B, H, N = c["seqs"], c["kv_heads"], max(s["new"])
    seq, position, at = token_rows(s)
    q = rotated(s, s["q"], position).float()
    q = q.gather(2, s["reorder_k"].long().repeat_interleave(Hq // H, 0).expand(T, Hq, D))
    qp = torch.zeros(B, N, Hq, D, device="cuda")
    qp[seq, at] = q
    qp = qp.transpose(1, 2).reshape(B, H, Hq // H * N, D)
    K = held_values(s, "k")
    score = torch.matmul(qp, K.transpose(2, 3)).mul_(s["sm_scale"])
    del K
    score = score.view(B, Hq, N, -1)
    t = torch.arange(score.shape[3], device="cuda")
    limit = s["lens"][:, None].long()
    if c["causal"]:
        n = (s["starts"][1:] - s["starts"][:-1])[:, None]
        limit = limit - n + 1 + torch.arange(N, device="cuda")
    score.masked_fill_((t >= limit[..., None])[:, None], -math.inf)
    m = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    V = held_values(s, "v")
    o = torch.matmul(p.view(B, H, -1, p.shape[-1]), torch.where((t < s["lens"][:, None])[:, None, :, None], V, torch.zeros((), device="cuda")))
    o = o.view(B, Hq, N, D) / torch.where(total == 0, torch.ones_like(total), total)
    o = o.transpose(1, 2)[seq, at]
    back = s["reorder_v"].long().repeat_interleave(Hq // H, 0).expand(T, Hq, D)
    return torch.empty_like(s["q"]).scatter_(2, back, o.to(s["q"].dtype))


def run(state):
    s, c = state, state["c"]
    if c["op"] == "rope":
        if own:
            q, k = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"), torch.empty(s["k"].shape, dtype=s["k"].dtype, device="cuda")
            s["rope"].apply(s["positions"], s["q"], q, s["k"], k, inverse=c["inverse"])
            return {"q": q, "k": k}
        cs = s["table"][s["positions"].long()]
        return {n: rotate(s[n], cs, c["rot_dim"], c["interleaved"], c["inverse"]) for n in ("q", "k")}
    if c["op"] == "append":
        if own:
            s["cache"].append(s["batch"], s["k"], s["v"], rope=s["rope"])
            k, v = s["cache"].read(s["batch"], window=False)
            return {"k": k, "v": v, "k_win": s["k_win"], "v_win": s["v_win"]}
        return plain_append(s)
    if own:
        return s["cache"].attention(s["batch"], s["q"], s["sm_scale"], causal=c["causal"], rope=s["rope"])
    return plain_attention(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact_rotation(x, cs, c, inverse=False):
    """The rotation as complex numbers, x [n, H, D] in 64 bits."""
    w = torch.complex(cs[..., 0].double(), cs[..., 1].double())[:, None]
    if inverse:
        w = w.conj()
    r, half = c["rot_dim"], c["rot_dim"] // 2
    first, second = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, half), slice(half, r))
    y = x.double().clone()
    turned = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * w
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "rope":
        cs = s["table"][s["positions"].long()]
        return {n: exact_rotation(s[n], cs, c, c["inverse"]) for n in ("q", "k")}
    W, H, D, G = c["window"], c["kv_heads"], c["head_dim"], c["group"]
    if c["op"] == "append":
        ends = [sum(s["new"][:b + 1]) for b in range(c["seqs"])]
        ring = {"k": s["k_win"].double(), "v": s["v_win"].double()}
        value = {}
        for name in ("k", "v"):
            value[name] = torch.empty(s["k"].shape, dtype=torch.float64, device="cuda")
            inverse = s["reorder_" + name].long().argsort(1)
            for b, (n, L, end) in enumerate(zip(s["new"], s["total"], ends)):
                x = s[name][end - n:end]
                if name == "k" and c["rot_dim"]:
                    # rotated keys are held in the tensor's type
                    x = exact_rotation(x, s["table"][L - n:L], c).to(x.dtype)
                xr = torch.stack([x[:, h][:, s["reorder_" + name][h].long()] for h in range(H)], 1).double()
                xg = xr.view(n, H, D // G, G)
                a = s["alpha"].double()
                lo, hi = xg.min(-1).values * a, xg.max(-1).values * a
                step, zero = ((hi - lo) / 15).half().double()[..., None], lo.half().double()[..., None]
                code = ((xg - zero) / step).round().clamp(0, 15)
                code = torch.where(step == 0, torch.zeros_like(code), code)
                v = (step * code + zero).view(n, H, D)
                value[name][end - n:end] = torch.stack([v[:, h][:, inverse[h]] for h in range(H)], 1)
                for t in range(max(L - W, L - n), L):
                    ring[name][b, :, t % W] = xr[t - (L - n)]
        return {"k": value["k"], "v": value["v"], "k_win": ring["k"], "v_win": ring["v"]}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    rep, end = c["q_heads"] // H, 0
    for b, (n, L) in enumerate(zip(s["new"], s["total"])):
        end += n
        q = s["q"][end - n:end]
        if c["rot_dim"]:
            # rotated queries are held in the tensor's type
            q = exact_rotation(q, s["table"][L - n:L], c).to(q.dtype)
        slots = s["page_table"][b, :-(-L // c["page"])].long()
        keep = torch.arange(L, device="cuda")[None] < (torch.arange(L - n, L, device="cuda")[:, None] + 1 if c["causal"] else L)
        for h in range(H):
            held = {}
            for name in ("k", "v"):
                codes = s[name + "_codes"][slots, h].reshape(-1, D // 2)[:L].int()
                meta = s[name + "_meta"][slots, h].reshape(-1, D // G, 2)[:L].double()
                x = torch.stack((codes % 16, codes // 16), 2).view(L, D // G, G).double() * meta[..., :1] + meta[..., 1:]
                x = x.view(L, D)
                recent = torch.arange(max(L - W, 0), L, device="cuda")
                if W:
                    x[recent] = s[name + "_win"][b, h, recent % W].double()
                held[name] = x[:, s["reorder_" + name][h].long().argsort()]
            rows = max(1, (1 << 28) // L // rep)
            for lo in range(0, n, rows):
                p = torch.einsum("nrd,td->rnt", q[lo:lo + rows, h * rep:(h + 1) * rep].double(), held["k"]) / math.sqrt(D)
                p = torch.softmax(p.masked_fill(~keep[lo:lo + rows], -math.inf), -1)
                out[end - n + lo:end - n + lo + p.shape[1], h * rep:(h + 1) * rep] = torch.einsum("rnt,td->nrd", p, held["v"])
    return out
