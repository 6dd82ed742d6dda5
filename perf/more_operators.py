"""Cases of the operators that shrink a paged cache by what attention looked at, and of rotations with several axes.

``own`` False: every operator in elementary torch operations, in 32 bits, rounded once at the end.  ``own`` True: the calls a
serving program makes of the library.  Shapes follow the benchmark workloads of this repository: 32 query heads over 32 or 8
KV heads of 128 channels, contexts of 4096 to 131072 tokens, groups of 32, 64 and 128 channels, windows of 128 and 256 tokens,
the ragged serving mix of 64 sequences with 1024 to 16384 tokens; keys with outlier channels.

A case's sequence lengths follow from its sizes alone (the seed makes the values), so that ``work`` is exact.

Definitions.

Rotation with several axes: every token has a position on each of A axes (time, height, width); pair j of a head turns by the
angle of row position[axis[j]] of the table: y1 = x1 c - x2 s, y2 = x2 c + x1 s in fp32, the products rounded, then the sum,
then to the tensor's type.  Backward: the same with -s.

Attention weights: w_out[t] = (t < L - n ? w[t] : 0) + sum over the new tokens' rows r of a KV head (its query heads; the last
``last`` tokens only, where that is not 0) that see token t of exp(sm_scale q'_r . K~_t - lse_r), K~ the cache's key: codes
h code + z, the newest ``window`` tokens unquantized from the ring.  lse is the row's logarithm of the softmax denominator, as
attention gives it.

Eviction: of L tokens a KV head keeps ``keep``: the ``first`` oldest, the ``recent`` newest, and of those between them the ones
with the largest weights (the lower token number where weights are equal).  Rows of keys, values and weights move together,
in the order they had; the ring follows.
"""
import math
import random

import torch

own = False

OUTLIERS, OUTLIER_SCALE = 4, 15.0
DTYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def axes(name, tokens, heads, head_dim, rot_dim, sections, layout, interleaved, inverse, dtype, context):
    return {"name": name, "op": "axes", "tokens": tokens, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "rot_dim": rot_dim,
            "sections": sections, "layout": layout, "interleaved": interleaved, "inverse": inverse, "dtype": dtype, "context": context}


def weights(name, seqs, new, prior, heads, head_dim, group, window, page, rot_dim, interleaved, dtype, causal=True, last=0):
    return {"name": name, "op": "weights", "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "prior_lo": prior[0], "prior_hi": prior[1],
            "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "group": group, "window": window, "page": page,
            "rot_dim": rot_dim, "interleaved": interleaved, "dtype": dtype, "causal": causal, "last": last}


def evict(name, seqs, length, keep, first, recent, heads, head_dim, group, window, page, dtype):
    return {"name": name, "op": "evict", "seqs": seqs, "new_lo": 0, "new_hi": 0, "prior_lo": length[0], "prior_hi": length[1], "keep": keep,
            "first": first, "recent": recent, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "group": group,
            "window": window, "page": page, "dtype": dtype}


def listed():
    return [
        # one decode step of the serving mix, text and images: 64 tokens, time, height and width in runs of 16, 24 and 24 pairs
        axes("axes decode", 64, (32, 8), 128, 128, "16 24 24", "runs", False, False, "bfloat16", 16384),
        # a prompt of 32k tokens, mostly image patches; the axes take turns among the pairs
        axes("axes prompt", 32768, (32, 8), 128, 128, "24 20 20", "turns", False, False, "float16", 32768),
        # gradients of a two-axis rotation of half the head in neighbouring pairs, an odd number of tokens, full precision
        axes("axes backward partial", 8191, (32, 32), 128, 64, "16 16", "runs", True, True, "float32", 16384),
        # one query over 4096 tokens, the smallest context of the benchmark: latency counts
        weights("weights short", 1, (1, 1), (4095, 4095), (32, 32), 128, 128, 128, 64, 128, False, "float16"),
        # a decode step of the serving mix: what each of 64 queries looked at is added to its sequence's weights
        weights("weights serving", 64, (1, 1), (1023, 16383), (32, 32), 128, 64, 256, 64, 128, False, "float16"),
        # a decode step over long contexts, grouped-query shape with fine groups
        weights("weights long", 4, (1, 1), (131071, 131071), (32, 8), 128, 32, 128, 64, 128, False, "bfloat16"),
        # a chunk of a long prompt: 2048 queries over 32k tokens
        weights("weights chunk", 1, (2048, 2048), (30720, 30720), (32, 8), 128, 64, 256, 64, 128, False, "float16"),
        # ragged prompts from their first token, narrow heads
        weights("weights prompts", 9, (1, 4095), (0, 0), (32, 32), 64, 32, 128, 16, 64, False, "bfloat16"),
        # prompts of 8192 tokens judged by their last 32 queries alone
        weights("weights observed", 4, (8192, 8192), (0, 0), (32, 8), 128, 64, 128, 64, 128, True, "bfloat16", True, 32),
        # a prompt of 32k tokens shrinks to 2048 before decoding begins
        evict("evict prompt", 1, (32768, 32768), 2048, 4, 256, (32, 8), 128, 64, 256, 64, "float16"),
        # the serving mix is brought back to at most 2048 tokens a sequence; the shorter ones stay whole
        evict("evict serving", 64, (1024, 16384), 2048, 4, 512, (32, 32), 128, 64, 256, 64, "float16"),
        # half of four long contexts goes, odd lengths, narrow pages
        evict("evict long", 4, (131001, 131071), 65521, 16, 4097, (32, 8), 128, 32, 128, 16, "bfloat16"),
    ]


def log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = {"bytes": 1.3e9, "flops": 5.0e11, "scores": 1.6e9, "values": 3.0e9}
    while True:
        op = rng.choice(["axes", "weights", "weights", "evict"])
        dtype = rng.choice(["float16", "bfloat16"])
        head_dim = rng.choice([64, 128, 128])
        rot_dim = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
        inter = rng.random() < 0.5
        heads = rng.choice([(32, 32), (32, 8), (32, 16), (32, 4), (8, 8), (24, 8)])
        group = rng.choice([g for g in (32, 64, 128) if g <= head_dim])
        window, page = rng.choice([0, 128, 256]), rng.choice([16, 32, 64, 128])
        if op == "axes":
            n, left, parts = rng.randint(1, 4), rot_dim // 2, []
            for i in range(n - 1):
                parts.append(rng.randint(1, left - (n - 1 - i)))
                left -= parts[-1]
            c = axes("", log_int(rng, 1, 32768), heads, head_dim, rot_dim, " ".join(str(p) for p in parts + [left]), rng.choice(["runs", "turns"]),
                     inter, rng.random() < 0.4, rng.choice(["float16", "bfloat16", "float32"]), 32768)
        elif op == "weights":
            hi = rng.choice([1, 1, log_int(rng, 2, 16), log_int(rng, 17, 4096)])
            prior = log_int(rng, 1, 131072)
            prior = (0, 0) if hi > 1 and rng.random() < 0.3 else (prior // rng.choice([1, 2, 8]), prior)
            c = weights("", log_int(rng, 1, 64), (max(1, hi // rng.choice([1, 4, 64])), hi), prior, heads, head_dim, group, window, page,
                        rng.choice([0, rot_dim]), inter, dtype, rng.random() < 0.8, rng.choice([0, 0, 1, 16, 64]))
        else:
            length = log_int(rng, 2, 131072)
            keep = log_int(rng, 1, length)
            recent = rng.randint(0, keep)
            first = rng.randint(0, min(16, keep - recent))
            c = evict("", log_int(rng, 1, 64), (max(1, length // rng.choice([1, 2, 16])), length), keep, first, recent, heads, head_dim, group,
                      0 if window > recent else window, page, dtype)
        del c["name"]
        w = work(c)
        values = scores = 0
        if op != "axes":
            new, total = lengths(c)
            values = len(total) * max(total) * heads[1] * (head_dim if op == "weights" else 8)
            scores = len(total) * max(new) * max(total) * heads[0]
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and scores <= most["scores"] and values <= most["values"]:
            return c


def lengths(c):
    """New tokens and total length of every sequence: from the case's sizes alone."""
    r = random.Random("%d %d %d %d %d" % (c["seqs"], c["new_lo"], c["new_hi"], c["prior_lo"], c["prior_hi"]))
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["seqs"])]
    return new, [n + r.randint(c["prior_lo"], c["prior_hi"]) for n in new]


def pair_axes(c):
    """The axis of every pair: runs of pairs in order, or taking turns until an axis has no pairs left."""
    parts = [int(x) for x in c["sections"].split()]
    if c["layout"] == "runs":
        return [a for a, n in enumerate(parts) for _ in range(n)]
    out, left = [], list(parts)
    while any(left):
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return out


def counted(c, n):
    return min(n, c["last"]) if c["last"] else n


def work(case):
    c = case
    D, H = c["head_dim"], c["kv_heads"]
    if c["op"] == "axes":
        n = c["tokens"] * (c["q_heads"] + H)
        elt, n_axes = (4 if c["dtype"] == "float32" else 2), len(c["sections"].split())
        return {"bytes": 2 * n * D * elt + c["tokens"] * (4 * c["rot_dim"] + 4 * n_axes), "flops": 3 * n * c["rot_dim"]}
    new, total = lengths(c)
    W, row = c["window"], D // 2 + 4 * (D // c["group"])      # one token's codes and parameters, keys or values
    if c["op"] == "weights":
        held = pairs = rows = 0
        for n, L in zip(new, total):
            m = counted(c, n)
            rows += m
            pairs += m * L - m * (m - 1) // 2 if c["causal"] else m * L
            held += H * (max(L - W, 0) * row + min(L, W) * D * 2) + 4 * H * (2 * L - n)      # keys; weights in and out
        return {"bytes": held + rows * (c["q_heads"] * (D * 2 + 4) + 4 * c["rot_dim"]), "flops": (2 * D + 2) * c["q_heads"] * pairs}
    moved = sum(min(L, c["keep"]) for L in total) * H
    ring = sum(min(L, W + 8, c["recent"] if L > c["keep"] else L) for L in total) * H if W else 0
    # weights read; rows of keys and values in and out; weights and numbers of the kept out; ring rows in and out
    return {"bytes": 4 * H * sum(total) + moved * (4 * row + 8) + ring * 2 * 2 * 2 * D, "flops": H * sum(total)}


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


def quantize(x, group):
    """fp32 x [..., D] -> codes uint8 [..., D] and fp16 parameters [..., D / group, 2] {h, z}."""
    xg = x.unflatten(-1, (-1, group))
    lo, hi = xg.amin(-1), xg.amax(-1)
    meta = torch.stack(((hi - lo) / 15.0, lo), -1).half()
    h, z = meta[..., 0:1].float(), meta[..., 1:2].float()
    codes = torch.where(h != 0, torch.round((xg - z) / h).clamp(0, 15), torch.zeros_like(xg))
    return codes.to(torch.uint8).flatten(-2), meta


def image_positions(T, n_axes):
    """Text and pictures in turn, as a prompt has them: runs of 40 text tokens (the same position on every axis), then a picture
    of 24 x 24 patches at one time, rows and columns on the second and third axis; the text goes on behind its largest position."""
    t = torch.arange(T, device="cuda")
    run, at = t // 616, t % 616
    base, patch = run * 64, at - 40
    grid = torch.stack((torch.zeros_like(t), patch // 24, patch % 24, patch % 7), 0)[:n_axes]
    return torch.where(at < 40, base + at, base + 40 + grid).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t = DTYPES[c["dtype"]]
    D, H, Hq = c["head_dim"], c["kv_heads"], c["q_heads"]
    s = {"c": c}
    if c["op"] == "axes":
        T, of_pair = c["tokens"], pair_axes(c)
        n_axes = max(of_pair) + 1
        # queries, keys and values of a layer lie side by side, as one projection writes them
        qkv = torch.randn(T, Hq + 2 * H, D, generator=g, device="cuda").to(t)
        s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + H]
        if T <= 256:
            s["positions"] = torch.randint(0, c["context"], (n_axes, T), generator=g, device="cuda", dtype=torch.int32)
        else:
            s["positions"] = (image_positions(T, n_axes) + torch.randint(0, 64, (1,), generator=g, device="cuda", dtype=torch.int32)) % c["context"]
        s["table"] = angles(c["context"], c["rot_dim"])
        s["axis"] = torch.tensor(of_pair, device="cuda")
        if own:
            from paper_2405_06219_b200 import binding
            s["rope"] = binding.RopeTable(s["table"], c["rot_dim"], c["interleaved"])
            s["axes"] = binding.RopeAxes(of_pair)
        return s
    new, total = lengths(c)
    T, P, W, seqs = sum(new), c["page"], c["window"], c["seqs"]
    held = [-(-n // P) for n in total]
    kept = [-(-min(n, c["keep"]) // P) for n in total] if c["op"] == "evict" else []
    n_pages = sum(held) + sum(kept) + 3
    # the pages that eviction moves rows to are the pool's last ones
    n_held = n_pages - sum(kept)
    for name, counts, lo, hi in (("page_table", held, 0, n_held), ("table_out", kept, n_held, n_pages)):
        order = (torch.randperm(hi - lo, generator=g, device="cuda") + lo).to(torch.int32)
        s[name] = torch.zeros(seqs, max(counts, default=1), dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(counts):
            s[name][b, :n] = order[at:at + n]
            at += n
    s["n_held"] = n_held
    s["lens"] = torch.tensor(total, dtype=torch.int32, device="cuda")
    s["starts"] = torch.tensor([sum(new[:b]) for b in range(seqs + 1)], dtype=torch.int32, device="cuda")
    s["new"], s["total"] = new, total
    s["capacity"] = max(total) + 5
    ng = D // c["group"]
    shape = (n_pages, H, P)
    if c["op"] == "evict":
        # rows are moved as they are: any bytes will do
        s["k_codes"], s["v_codes"] = (torch.randint(0, 256, (*shape, D // 2), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        s["k_meta"], s["v_meta"] = (torch.rand(*shape, ng, 2, generator=g, device="cuda").half() for _ in range(2))
        s["ring"], s["slots"] = W + 8 if W else 0, torch.arange(seqs, dtype=torch.int32, device="cuda")
        s["slots_out"] = s["slots"] + seqs
        s["k_win"], s["v_win"] = (torch.randn(2 * seqs, H, s["ring"], D, generator=g, device="cuda").to(t) for _ in range(2))
        # a few tokens hold most of what was looked at, many share the smallest weights
        w = torch.exp(2.0 * torch.randn(2 * seqs, H, s["capacity"], generator=g, device="cuda"))
        s["weights"] = torch.floor(w * 64.0) / 64.0
        s["weights_out"] = torch.zeros_like(s["weights"])
        if own:
            from paper_2405_06219_b200 import binding
            s["cache"] = binding.SkvqPagedCache(
                Hq, H, D, c["group"], W, P, n_pages, 2 * seqs, dtype=t, ring_tokens=s["ring"],
                buffers={n: s[n] for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")})
            s["batch"] = s["cache"].batch(s["page_table"], s["lens"], s["starts"], n_tokens=0, max_new=0, max_len=max(total), slots=s["slots"])
        return s
    sigma = key_sigma(g, H, D)
    s["reorder_k"] = sigma.argsort(1).to(torch.int32)
    s["sm_scale"] = 1.0 / math.sqrt(D)
    s["table"] = angles(max(total), c["rot_dim"]) if c["rot_dim"] else None
    sigma_r = sigma.gather(1, s["reorder_k"].long())
    s["k_codes"] = torch.zeros(*shape, D // 2, dtype=torch.uint8, device="cuda")
    s["k_meta"] = torch.zeros(*shape, ng, 2, dtype=torch.float16, device="cuda")
    step = max(1, (1 << 27) // (H * P * D))
    for lo in range(0, n_pages, step):
        n = min(step, n_pages - lo)
        x = (torch.randn(n, H, P, D, generator=g, device="cuda") * sigma_r[None, :, None]).to(t).float()
        codes, meta = quantize(x, c["group"])
        s["k_codes"][lo:lo + n] = codes[..., 0::2] | codes[..., 1::2] << 4
        s["k_meta"][lo:lo + n] = meta
    s["k_win"] = (torch.randn(seqs, H, W, D, generator=g, device="cuda") * sigma_r[None, :, None]).to(t)
    # with the keys' outliers, scores up to 10 or 20
    s["q"] = (0.5 * torch.randn(T, Hq, D, generator=g, device="cuda")).to(t)
    s["weights"] = torch.rand(seqs, H, s["capacity"], generator=g, device="cuda") ** 8
    s["weights_out"] = torch.zeros_like(s["weights"])
    s["lse"] = torch.cat([denominators(s, b) for b in range(seqs)])
    if own:
        from paper_2405_06219_b200 import binding
        buffers = {n: s[n] for n in ("k_codes", "k_meta", "k_win")}
        buffers.update({"v" + n[1:]: torch.zeros_like(x) for n, x in buffers.items()})
        s["cache"] = binding.SkvqPagedCache(Hq, H, D, c["group"], W, P, n_pages, seqs, dtype=t, reorder_k=s["reorder_k"], buffers=buffers)
        s["batch"] = s["cache"].batch(s["page_table"], s["lens"], s["starts"], n_tokens=T, max_new=max(new), max_len=max(total))
        s["rope"] = binding.RopeTable(s["table"], c["rot_dim"], c["interleaved"]) if c["rot_dim"] else None
    return s


def denominators(s, b):
    """lse [n, Hq] of one sequence's rows, as attention of this step gives it."""
    c = s["c"]
    n, L, end = s["new"][b], s["total"][b], sum(s["new"][:b + 1])
    H, Hq, D = c["kv_heads"], c["q_heads"], c["head_dim"]
    q = rotated(s, s["q"][end - n:end], torch.arange(L - n, L, device="cuda")).float()
    q = q.gather(2, s["reorder_k"].long().repeat_interleave(Hq // H, 0).expand(n, Hq, D)).transpose(0, 1)      # [Hq, n, D]
    K = held_keys(s, [b])[0]                                                                                  # [H, L', D]
    t = torch.arange(K.shape[1], device="cuda")
    out = torch.empty(n, Hq, device="cuda")
    rows = max(1, (1 << 28) // (K.shape[1] * Hq))
    for lo in range(0, n, rows):
        m = min(rows, n - lo)
        x = torch.matmul(q[:, lo:lo + m].reshape(H, Hq // H * m, D), K.transpose(1, 2)).view(Hq, m, -1) * s["sm_scale"]
        limit = L - n + 1 + torch.arange(lo, lo + m, device="cuda") if c["causal"] else torch.full((m,), L, device="cuda")
        x.masked_fill_(t >= limit[:, None], -math.inf)
        out[lo:lo + m] = torch.logsumexp(x, -1).t()
    return out


# ------------------------------------------------------------------------------------------------ plain forms
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


def rotated(s, x, position):
    c = s["c"]
    return rotate(x, s["table"][position], c["rot_dim"], c["interleaved"]) if c["rot_dim"] else x


def axis_angles(s):
    """fp32 [T, pairs, 2]: pair j of token t from row positions[axis[j], t]."""
    row = s["positions"].long()[s["axis"]].t()                                    # [T, pairs]
    return s["table"][row, torch.arange(row.shape[1], device="cuda")]


def held_keys(s, seqs):
    """The keys of some sequences as fp32 [n, H, Lmax, D], reordered channels: pages, the window's tokens from the ring."""
    c = s["c"]
    W, P = c["window"], c["page"]
    pages = -(-max(s["total"][b] for b in seqs) // P)
    ids = s["page_table"][seqs, :pages].long()
    codes = s["k_codes"][ids].transpose(1, 2).flatten(2, 3)      # [n, H, L, D / 2]
    meta = s["k_meta"][ids].transpose(1, 2).flatten(2, 3).float()
    x = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).unflatten(-1, (-1, c["group"])).float()
    x = x.mul_(meta[..., 0:1]).add_(meta[..., 1:2]).flatten(-2)
    if W:
        lens = s["lens"][seqs].long()
        t = lens[:, None] - W + torch.arange(W, device="cuda")
        i = torch.arange(len(seqs), device="cuda")[:, None].expand_as(t)
        i, t = i[t >= 0], t[t >= 0]
        x[i, :, t] = s["k_win"][torch.tensor(seqs, device="cuda")[i], :, t % W].float()
    return x


def plain_weights(s):
    c = s["c"]
    T, Hq, D = s["q"].shape
    B, H = c["seqs"], c["kv_heads"]
    n = (s["starts"][1:] - s["starts"][:-1]).long()
    m = n.clamp(max=c["last"]) if c["last"] else n
    N = max(counted(c, x) for x in s["new"])
    # the counted rows, a sequence's last m, padded to N
    i = torch.arange(N, device="cuda")
    real = i < m[:, None]
    row = torch.where(real, s["starts"][1:].long()[:, None] - m[:, None] + i, torch.zeros_like(i))
    position = s["lens"].long()[:, None] - m[:, None] + i
    q = rotated(s, s["q"][row].flatten(0, 1), position.clamp(0, max(s["total"]) - 1).flatten()).float()
    q = q.gather(2, s["reorder_k"].long().repeat_interleave(Hq // H, 0).expand(B * N, Hq, D))
    q = q.view(B, N, Hq, D).transpose(1, 2).reshape(B, H, Hq // H * N, D)
    score = torch.matmul(q, held_keys(s, list(range(B))).transpose(2, 3)).mul_(s["sm_scale"]).view(B, Hq, N, -1)
    t = torch.arange(score.shape[3], device="cuda")
    limit = position + 1 if c["causal"] else s["lens"].long()[:, None].expand(B, N)
    lse = s["lse"][row]                                                            # [B, N, Hq]
    out_of = (t >= limit[..., None])[:, None] | ~(real[..., None] & torch.isfinite(lse)).transpose(1, 2)[..., None]
    p = score.sub_(lse.transpose(1, 2)[..., None]).masked_fill_(out_of, -math.inf).exp_()
    total = p.view(B, H, -1, p.shape[3]).sum(2)
    L = min(total.shape[2], s["capacity"])
    old = torch.where((t[:L] < (s["lens"].long() - n)[:, None])[:, None], s["weights"][:, :, :L], torch.zeros((), device="cuda"))
    out = s["weights_out"]
    out[:, :, :L] = torch.where((t[:L] < s["lens"][:, None])[:, None], old + total[:, :, :L], out[:, :, :L])
    return out


def plain_evict(s):
    c = s["c"]
    B, H, P, keep, D = c["seqs"], c["kv_heads"], c["page"], c["keep"], c["head_dim"]
    lens = s["lens"].long()
    left = lens.clamp(max=keep)
    whole = lens <= keep
    L = max(s["total"])
    t = torch.arange(L, device="cuda")
    w = s["weights"][s["slots"].long(), :, :L]
    always = (t < c["first"]) | (t >= lens[:, None] - c["recent"]) | whole[:, None]
    w = torch.where(always[:, None], torch.full((), math.inf, device="cuda"), w)
    w = torch.where((t < lens[:, None])[:, None], w, torch.full((), -math.inf, device="cuda"))
    ranked = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    i = torch.arange(ranked.shape[-1], device="cuda")
    mine = (i < left[:, None])[:, None]
    kept = torch.where(mine, ranked, torch.full((), 1 << 40, device="cuda")).sort(-1).values
    kept = torch.where(mine, kept, torch.full((), -1, device="cuda"))
    b, h, r = torch.nonzero(kept >= 0, as_tuple=True)
    old = kept[b, h, r]
    src, dst = s["page_table"][b, old // P].long(), s["table_out"][b, r // P].long()
    for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
        x = s[name]
        x[dst, h, r % P] = x[src, h, old % P]
    s["weights_out"][s["slots_out"][b].long(), h, r] = s["weights"][s["slots"][b].long(), h, old]
    R, gone = s["ring"], lens - left
    ring_from = torch.zeros(B, dtype=torch.int64, device="cuda")
    if R:
        rows = torch.where(whole, torch.full((), R, device="cuda"), torch.full((), min(R, c["recent"]), device="cuda"))
        ring_from = (lens - rows).clamp(min=0) - gone
        k = torch.arange(R, device="cuda")
        b, k = torch.nonzero((k < left[:, None] - ring_from[:, None]), as_tuple=True)
        to = ring_from[b] + k
        for name in ("k_win", "v_win"):
            s[name][s["slots_out"][b].long(), :, to % R] = s[name][s["slots"][b].long(), :, (to + gone[b]) % R]
    full = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
    full[..., :kept.shape[-1]] = kept.to(torch.int32)
    return evicted(s, full, left.to(torch.int32))


def evicted(s, kept, lens):
    # what was written: the pages, the slots' weights and their rings
    return {"kept": kept, "lens": lens, "weights": s["weights_out"][s["c"]["seqs"]:],
            **{n: s[n][s["n_held"]:] for n in ("k_codes", "v_codes", "k_meta", "v_meta")},
            **{n: s[n][s["c"]["seqs"]:] for n in ("k_win", "v_win")}}


def run(state):
    s, c = state, state["c"]
    if c["op"] == "axes":
        if own:
            q, k = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"), torch.empty(s["k"].shape, dtype=s["k"].dtype, device="cuda")
            s["rope"].apply_axes(s["axes"], s["positions"], s["q"], q, s["k"], k, inverse=c["inverse"])
            return {"q": q, "k": k}
        cs = axis_angles(s)
        return {n: rotate(s[n], cs, c["rot_dim"], c["interleaved"], c["inverse"]) for n in ("q", "k")}
    if c["op"] == "weights":
        if own:
            return s["cache"].accumulate_weights(s["batch"], s["q"], s["lse"], s["weights"], s["sm_scale"], out=s["weights_out"],
                                                 causal=c["causal"], rope=s["rope"], last=c["last"])
        return plain_weights(s)
    if own:
        kept, lens, _ = s["cache"].evict(s["batch"], s["weights"], c["keep"], first=c["first"], recent=c["recent"], weights_out=s["weights_out"],
                                         page_table_out=s["table_out"], slots_out=s["slots_out"])
        return evicted(s, kept, lens)
    return plain_evict(s)


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
    if c["op"] == "axes":
        of_pair = pair_axes(c)
        cs = torch.stack([s["table"][s["positions"][a].long(), j] for j, a in enumerate(of_pair)], 1)
        return {n: exact_rotation(s[n], cs, c, c["inverse"]) for n in ("q", "k")}
    H, D, G, P, W = c["kv_heads"], c["head_dim"], c["group"], c["page"], c["window"]
    if c["op"] == "evict":
        return exact_evict(s)
    out = s["weights_out"].double()
    rep, end = c["q_heads"] // H, 0
    for b, (n, L) in enumerate(zip(s["new"], s["total"])):
        end += n
        m = counted(c, n)
        q = s["q"][end - m:end]
        if c["rot_dim"]:
            # rotated queries are held in the tensor's type
            q = exact_rotation(q, s["table"][L - m:L], c).to(q.dtype)
        slots = s["page_table"][b, :-(-L // P)].long()
        for h in range(H):
            codes = s["k_codes"][slots, h].reshape(-1, D // 2)[:L].int()
            meta = s["k_meta"][slots, h].reshape(-1, D // G, 2)[:L].double()
            x = torch.stack((codes % 16, codes // 16), 2).view(L, D // G, G).double() * meta[..., :1] + meta[..., 1:]
            x = x.view(L, D)
            recent = torch.arange(max(L - W, 0), L, device="cuda")
            if W:
                x[recent] = s["k_win"][b, h, recent % W].double()
            key = x[:, s["reorder_k"][h].long().argsort()]
            out[b, h, :L] = 0
            out[b, h, :L - n] = s["weights"][b, h, :L - n].double()
            rows = max(1, (1 << 27) // L // rep)
            for lo in range(0, m, rows):
                part = q[lo:lo + rows, h * rep:(h + 1) * rep].double()
                p = torch.einsum("nrd,td->rnt", part, key) / math.sqrt(D)
                p = torch.exp(p - s["lse"][end - m + lo:end - m + lo + part.shape[0], h * rep:(h + 1) * rep].double().t()[..., None])
                if c["causal"]:
                    last = torch.arange(L - m + lo, L - m + lo + part.shape[0], device="cuda")
                    p *= torch.arange(L, device="cuda")[None] <= last[:, None]
                out[b, h, :L] += p.sum((0, 1))
    return out


def exact_evict(s):
    c = s["c"]
    H, P, W, keep, R = c["kv_heads"], c["page"], c["window"], c["keep"], s["ring"]
    kept = torch.full((c["seqs"], H, keep), -1, dtype=torch.int32, device="cuda")
    after = {n: s[n].clone() for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")}
    weights_out, lens = s["weights_out"].clone(), []
    for b, L in enumerate(s["total"]):
        n = min(L, keep)
        lens.append(n)
        for h in range(H):
            chosen = torch.ones(L, dtype=torch.bool, device="cuda")
            if L > keep:
                lo, hi = c["first"], L - c["recent"]
                w = s["weights"][b, h, lo:hi].double()
                count = keep - c["first"] - c["recent"]
                best = torch.argsort(-w, stable=True)[:count]
                chosen[lo:hi] = False
                chosen[lo + best] = True
            ids = torch.nonzero(chosen)[:, 0]
            kept[b, h, :n] = ids.to(torch.int32)
            weights_out[c["seqs"] + b, h, :n] = s["weights"][b, h, ids]
            row = torch.arange(n, device="cuda")
            for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
                after[name][s["table_out"][b, row // P].long(), h, row % P] = s[name][s["page_table"][b, ids // P].long(), h, ids % P]
        if W:
            live = min(R, L if L <= keep else c["recent"], L)
            old = torch.arange(L - live, L, device="cuda")
            for name in ("k_win", "v_win"):
                after[name][c["seqs"] + b][:, (old - (L - n)) % R] = s[name][b][:, old % R]
    return evicted({**after, "c": c, "n_held": s["n_held"], "weights_out": weights_out}, kept, torch.tensor(lens, dtype=torch.int32, device="cuda"))
