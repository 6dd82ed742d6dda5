"""Rotary positions, paged 4-bit append/read and attention on the GPU against the plain 64-bit forms of paged_reference.

Rotations, codes, parameters and ring rows are compared bit for bit with the documented fp32 roundings; attention against 64
bits with the error bound that Reference.attention counts out."""
import math
import random

import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build, workloads

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


def bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------------------ rotation
@pytest.mark.parametrize("first,n,rot,kind", [(0, 700, 128, 0), (1048000, 576, 64, 0), (2147483000, 640, 8, 0), (0, 1, 2, 0), (5, 100, 256, 3), (131000, 72, 128, 2)])
def test_table_is_right_to_fp32_at_far_positions(first, n, rot, kind):
    f, amp = B.skvq_rope_frequencies(rot, B.SkvqRopeScaling(kind, 4096, 10000.0, 8.0, 32.0, 1.0))
    table = torch.full((n + 2, rot // 2, 2), 7.0, device="cuda")
    B.skvq_rope_table(f, amp, first, n, table[1:])
    got = table.cpu()
    assert (got[0] == 7).all() and (got[-1] == 7).all()
    # the angle in 80-bit extended precision: position times frequency is exact there to 2^-33 radians at 2^31
    angle = np.arange(first, first + n).astype(np.longdouble)[:, None] * np.array(f, np.longdouble)
    want = np.stack((amp * np.cos(angle), amp * np.sin(angle)), -1).astype(np.float64)
    # half a step of fp32 at the amplitude (below 2), and the errors of the reference's own product
    assert np.abs(got[1:-1].numpy() - want).max() <= 2.0 ** -24 * max(1.0, amp) + 2.0 ** -32


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("T,Hq,Hk,D,rot,inter", [
    (1, 1, 0, 2, 2, False), (3, 4, 1, 128, 128, False), (67, 32, 8, 128, 128, True), (130, 5, 5, 64, 32, False), (33, 3, 2, 80, 48, True),
    (1000, 8, 2, 128, 64, True), (19, 2, 1, 96, 20, False), (7, 3, 3, 33, 30, True), (5, 2, 2, 512, 256, False), (260, 6, 2, 64, 16, False),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_bit_exact(dtype, T, Hq, Hk, D, rot, inter, inverse):
    g = gen(T * 7 + D)
    qkv = torch.randn(T, Hq + Hk + 1, D, generator=g).to(dtype)
    cs = ref.table64(rot, 500).float()
    pos = torch.randint(0, 500, (T,), generator=g, dtype=torch.int32)
    rope = B.RopeTable(cs.cuda(), rot, inter)
    dev = qkv.cuda()
    q, k = dev[:, :Hq], dev[:, Hq:Hq + Hk] if Hk else None
    q_out = torch.full((T, Hq, D), 3.0, dtype=dtype, device="cuda")
    k_out = torch.full((T, Hk, D), 3.0, dtype=dtype, device="cuda") if Hk else None
    rope.apply(pos.cuda(), q, q_out, k, k_out, inverse=inverse)
    want = ref.rotate32(qkv, cs[pos.long()], rot, inter, inverse)
    assert torch.equal(bits(q_out.cpu()), bits(want[:, :Hq]))
    if Hk:
        assert torch.equal(bits(k_out.cpu()), bits(want[:, Hq:Hq + Hk]))
    assert torch.equal(bits(dev.cpu()), bits(qkv))                                # the input is left alone
    # 64 bits: three roundings of 2^-24 of the terms, one of the type
    exact = ref.rotate(qkv[:, :Hq], cs[pos.long()], rot, inter, inverse)
    terms = qkv[:, :Hq].double().abs().amax(-1, keepdim=True) * 2
    assert ((q_out.cpu().double() - exact).abs() <= terms * 2.0 ** -23 + exact.abs() * torch.finfo(dtype).eps / 2 * 1.01 + 2.0 ** -25).all()
    rope.apply(pos.cuda(), q, None, k, None, inverse=inverse)                     # in place, inside the packed tensor
    assert torch.equal(bits(dev.cpu()[:, :Hq + Hk]), bits(want[:, :Hq + Hk])) and torch.equal(bits(dev.cpu()[:, -1]), bits(qkv[:, -1]))


def test_inverse_is_the_gradient_of_the_rotation():
    T, H, D, rot = 9, 3, 64, 48
    g = gen(5)
    x, dy = torch.randn(T, H, D, generator=g), torch.randn(T, H, D, generator=g)
    cs = ref.table64(rot, T).float()
    pos = torch.arange(T, dtype=torch.int32)
    rope = B.RopeTable(cs.cuda(), rot, True)
    dx = torch.empty(T, H, D, device="cuda")
    rope.apply(pos.cuda(), dy.cuda(), dx, inverse=True)
    x64 = x.double().requires_grad_()
    y = torch.zeros(T, H, D, dtype=torch.float64)
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double()
    y = torch.cat((torch.stack((x64[..., 0:rot:2] * c - x64[..., 1:rot:2] * s, x64[..., 1:rot:2] * c + x64[..., 0:rot:2] * s), -1).flatten(-2), x64[..., rot:]), -1)
    (y * dy.double()).sum().backward()
    assert (dx.cpu().double() - x64.grad).abs().max() <= 4 * float(dy.abs().max()) * 2.0 ** -24
    # differences of the forward rotation along random directions (the rotation is linear: one step is exact but for roundings)
    for seed in range(4):
        d = torch.randn(T, H, D, generator=gen(seed))
        out = [torch.empty(T, H, D, device="cuda") for _ in range(2)]
        rope.apply(pos.cuda(), (x + d).cuda(), out[0])
        rope.apply(pos.cuda(), (x - d).cuda(), out[1])
        diff = float((((out[0] - out[1]).cpu().double() / 2) * dy.double()).sum())
        want = float((dx.cpu().double() * d.double()).sum())
        n = T * H * D      # every term is off by a few roundings of values below 10
        assert abs(diff - want) <= n * 10 * float(dy.abs().max()) * 2.0 ** -22


def test_rotation_reports_positions_outside_the_table_and_leaves_their_rows():
    cs = ref.table64(64, 10).float()
    rope = B.RopeTable(cs.cuda(), 64)
    x = torch.randn(4, 2, 64).half()
    pos = torch.tensor([0, 10, -1, 9], dtype=torch.int32)
    out, status = torch.full((4, 2, 64), 5.0, dtype=F16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    rope.apply(pos.cuda(), x.cuda(), out, status=status)
    assert int(status.item()) == B.SKVQ_STATUS_BAD_POSITION
    assert (out.cpu()[1:3] == 5).all()
    want = ref.rotate32(x, cs[pos.long().clamp(0, 9)], 64, False)
    assert torch.equal(out.cpu()[[0, 3]], want[[0, 3]])


# ------------------------------------------------------------------------------------------------ the paged cache
class Paged:
    """A library cache and the plain reference side by side; every byte that holds nothing is poisoned."""

    def __init__(self, n_seqs=2, Hq=4, H=2, D=128, G=64, W=32, P=16, R=None, dtype=F16, rot=0, inter=False, reorder=True, seed=0, max_len=400,
                 spare=0, slots=None, outliers=True):
        g = gen(seed)
        self.g, self.n, self.Hq, self.H, self.D, self.P, self.dtype, self.W = g, n_seqs, Hq, H, D, P, dtype, W
        self.max_pages = -(-max_len // P)
        n_pages = n_seqs * self.max_pages + spare
        perm = [torch.stack([torch.randperm(D, generator=g) for _ in range(H)]).int() if reorder else None for _ in range(2)]
        alpha = [0.85 + 0.15 * torch.rand(H, D // G, generator=g) if reorder else None for _ in range(2)]
        self.table = ref.table64(rot, max_len).float() if rot else None
        self.rope = B.RopeTable(self.table.cuda(), rot, inter) if rot else None
        n_slots = n_seqs if slots is None else max(slots) + 1
        self.cache = B.SkvqPagedCache(Hq, H, D, G, W, P, n_pages, n_slots, dtype, *perm, *alpha, ring_tokens=R)
        for name in ("k_codes", "v_codes"):
            getattr(self.cache, name).fill_(0xFF)
        for name in ("k_meta", "v_meta", "k_win", "v_win"):
            getattr(self.cache, name).fill_(math.nan)
        self.ref = ref.Reference(n_seqs, Hq, H, D, G, W, dtype, *perm, *alpha, self.table, rot, inter)
        order = spare + torch.randperm(n_seqs * self.max_pages, generator=g)
        self.page_table = order.view(n_seqs, self.max_pages).int().cuda()
        self.slots = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
        self.scale = torch.exp(0.5 * torch.randn(H, D, generator=g))
        if outliers:
            self.scale[:, torch.randperm(D, generator=g)[:3]] *= 15

    def batch(self, new, lens, pad=0, max_new=None, max_len=None):
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        T = starts[-1] + pad
        return self.cache.batch(self.page_table, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                torch.tensor(starts, dtype=torch.int32, device="cuda"), T, max(new) if max_new is None else max_new,
                                max(max(lens), 1) if max_len is None else max_len, self.slots)

    def keys(self, T):
        return (torch.randn(T, self.H, self.D, generator=self.g) * self.scale).to(self.dtype), torch.randn(T, self.H, self.D, generator=self.g).to(self.dtype)

    def lens(self):
        return [len(r) for r in self.ref.rows]

    def append(self, new, pad=0):
        k, v = self.keys(sum(new) + pad)
        lens = [a + n for a, n in zip(self.lens(), new)]
        b = self.batch(new, lens, pad)
        self.cache.append(b, k.cuda(), v.cuda(), rope=self.rope)
        at = 0
        for i, n in enumerate(new):
            self.ref.append(i, k[at:at + n], v[at:at + n])
            at += n
        return b

    def check_rows(self):
        """Every token's codes, parameters and ring rows bit for bit; every other byte as it was."""
        torch.cuda.synchronize()
        c = self.cache
        pt = self.page_table.cpu().long()
        touched = torch.zeros(c.k_codes.shape[0], self.P, dtype=torch.bool)
        R = c.cfg.ring_tokens
        ring = torch.zeros(c.cfg.n_slots, max(R, 1), dtype=torch.bool)
        codes, meta, win = [getattr(c, "k_codes").cpu(), c.v_codes.cpu()], [c.k_meta.cpu(), c.v_meta.cpu()], [c.k_win.cpu(), c.v_win.cpu()]
        for b, rows in enumerate(self.ref.rows):
            L = len(rows)
            slot = b if self.slots is None else int(self.slots[b])
            for t, row in enumerate(rows):
                page, at = int(pt[b, t // self.P]), t % self.P
                touched[page, at] = True
                for s in range(2):
                    packed = row[2 + 2 * s][:, 0::2] | row[2 + 2 * s][:, 1::2] << 4
                    assert torch.equal(codes[s][page, :, at], packed), (b, t, s)
                    assert torch.equal(bits(meta[s][page, :, at]), bits(row[3 + 2 * s])), (b, t, s)
                    if self.W and t >= L - R:
                        ring[slot, t % R] = True
                        assert torch.equal(bits(win[s][slot, :, t % R]), bits(row[s])), (b, t, s)
        for s in range(2):
            assert (codes[s].permute(0, 2, 1, 3)[~touched] == 0xFF).all()
            assert torch.isnan(meta[s].transpose(1, 2)[~touched]).all()
            if self.W:
                assert torch.isnan(win[s].transpose(1, 2)[~ring]).all()

    def check_attention(self, new, lens=None, causal=True, pad=0, n_splits=0, sm_scale=None, lse=True, q=None, **kw):
        lens = self.lens() if lens is None else lens
        sm_scale = 1 / math.sqrt(self.D) if sm_scale is None else sm_scale
        T = sum(new)
        q = torch.randn(T + pad, self.Hq, self.D, generator=self.g).to(self.dtype) if q is None else q
        out = torch.full((T + pad, self.Hq, self.D), 9.0, dtype=self.dtype, device="cuda")
        ls = torch.full((T + pad, self.Hq), 9.0, device="cuda") if lse else None
        self.cache.attention(self.batch(new, lens, pad, **kw), q.cuda(), sm_scale, out=out, causal=causal, rope=self.rope, lse=ls, n_splits=n_splits)
        got, at = out.cpu().double(), 0
        assert (got[T:] == 9).all()
        for b, n in enumerate(new):
            want, wl, err, el = self.ref.attention(b, q[at:at + n], sm_scale, causal)
            bad = (got[at:at + n] - want).abs() - err
            assert not torch.isnan(got[at:at + n]).any() and (bad <= 0).all(), (b, float(bad.max()), float(err.max()))
            if lse:
                l = ls.cpu().double()[at:at + n]
                assert torch.equal(l == -math.inf, wl == -math.inf)
                fin = wl != -math.inf
                assert ((l - wl).abs()[fin] <= el[fin]).all(), (b, float(((l - wl).abs() - el)[fin].max()))
            at += n
        if lse:
            assert (ls.cpu()[T:] == 9).all()
        return out


SHAPES = [
    dict(D=128, G=64, H=2, Hq=4, P=16, W=32), dict(D=128, G=128, H=1, Hq=1, P=64, W=0, dtype=BF16), dict(D=128, G=32, H=2, Hq=2, P=32, W=20, R=33, rot=128),
    dict(D=64, G=32, H=3, Hq=9, P=16, W=16, rot=32, inter=True, dtype=BF16), dict(D=64, G=64, H=1, Hq=8, P=128, W=5, R=8, rot=64), dict(D=128, G=128, H=2, Hq=32, P=256, W=128, rot=20),
    dict(D=128, G=64, H=2, Hq=2, P=64, W=64, reorder=False, rot=128, inter=True, dtype=BF16),
]


@pytest.mark.parametrize("kw", SHAPES)
def test_append_and_read_bit_exact(kw):
    p = Paged(n_seqs=3, seed=11, spare=2, slots=[4, 0, 2], **kw)
    for new in ([17, 0, 1], [1, 1, 1], [130, 5, 64], [1, 1, 1], [0, 33, 0], [1, 90, 2]):
        b = p.append(new, pad=3)
        for window in (True, False):
            T = sum(new) + 3
            k, v = (torch.full((T, p.H, p.D), 9.0, dtype=p.dtype, device="cuda") for _ in range(2))
            p.cache.read(b, k, v, window=window)
            at = 0
            for i, n in enumerate(new):
                L = len(p.ref.rows[i])
                for got, which, idx in ((k, "k", p.ref.rk), (v, "v", p.ref.rv)):
                    want = torch.empty(n, p.H, p.D, dtype=p.dtype)
                    val = p.ref.values(i, which, window)[L - n:].float().to(p.dtype)
                    for h in range(p.H):
                        want[:, h, idx[h]] = val[:, h]
                    assert torch.equal(bits(got[at:at + n].cpu()), bits(want)), (i, which, window)
                at += n
            assert (k[sum(new):] == 9).all() and (v[sum(new):] == 9).all()
    p.check_rows()
    assert int(p.cache.status[0]) == 0


def test_paged_rows_equal_the_contiguous_cache():
    """The same keys and values appended to SkvqCache at 4 bits: the same zero points; the steps differ by one fp16 step at most
    (the quotient by 15 against the product with 1/15), and where they are the same, so are the codes."""
    w = workloads.configs()[4].scaled(batch=2, context=300, ragged=None, n_q_heads=4, n_kv_heads=4, window=0)
    flat = B.SkvqCache.for_workload(w, 300)
    k, v = torch.from_numpy(w.prefill("k", 300)).cuda(), torch.from_numpy(w.prefill("v", 300)).cuda()
    flat.append(k, v)
    cache = B.SkvqPagedCache(4, 4, 128, 64, 0, 64, 10, 2, reorder_k=w.reorder_index("k"), reorder_v=w.reorder_index("v"), alpha_k=w.alphas(), alpha_v=w.alphas())
    pt = torch.tensor([[9, 1, 7, 3, 5], [0, 2, 4, 6, 8]], dtype=torch.int32, device="cuda")
    lens, starts = torch.tensor([300, 300], dtype=torch.int32, device="cuda"), torch.tensor([0, 300, 600], dtype=torch.int32, device="cuda")
    batch = cache.batch(pt, lens, starts, 600, 300, 300)
    cache.append(batch, k.reshape(600, 4, 128), v.reshape(600, 4, 128))
    for side in "kv":
        (ac, bc), (am, bm) = [(getattr(flat, side + n)[:, :, :300].cpu(), getattr(cache, side + n)[pt.long()].transpose(1, 2).flatten(2, 3)[:, :, :300].cpu())
                              for n in ("_codes", "_meta")]
        am, bm = bits(am).int(), bits(bm).int()
        assert torch.equal(am[..., 1], bm[..., 1]) and (am[..., 0] - bm[..., 0]).abs().max() <= 1
        same = (am[..., 0] == bm[..., 0]).all(-1)
        assert same.float().mean() > 0.99 and torch.equal(ac[same], bc[same])
    q = torch.from_numpy(w.query(0)).cuda()
    one = cache.batch(pt, lens, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), 2, 1, 300)
    a, b = flat.attention(q, w.sm_scale, 300), cache.attention(one, q, w.sm_scale)
    assert (a.float() - b.float()).abs().max() <= 4e-3      # each is within 2e-3 of the exact value


@pytest.mark.parametrize("kw", SHAPES)
@pytest.mark.parametrize("n_splits", [0, 3])
def test_single_token_attention(kw, n_splits):
    p = Paged(n_seqs=4, seed=21, **kw)
    p.append([1, 300, 33, 0])
    p.check_attention([1, 1, 1, 0], n_splits=n_splits)
    p.append([1, 1, 1, 1])
    p.check_attention([1, 1, 1, 1], n_splits=n_splits)
    assert int(p.cache.status[0]) == 0


@pytest.mark.parametrize("kw", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_several_rows(kw, causal):
    p = Paged(n_seqs=4, seed=31, **kw)
    p.append([70, 129, 5, 200])
    p.check_attention([4, 7, 5, 1], causal=causal, pad=2)
    p.append([3, 2, 16, 17])
    p.check_attention([3, 2, 16, 17], causal=causal)
    p.check_attention([0, 0, 21, 0], causal=causal)


@pytest.mark.parametrize("kw", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_prompts_and_chunks(kw, causal):
    p = Paged(n_seqs=3, seed=41, **kw)
    p.append([150, 1, 77])
    p.check_attention([150, 1, 77], causal=causal, pad=5)
    p.append([130, 200, 64])
    p.check_attention([130, 200, 64], causal=causal)


@pytest.mark.parametrize("lens", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_lengths_around_every_boundary(lens):
    p = Paged(n_seqs=1, Hq=2, H=1, D=64, G=32, W=16, P=16, seed=lens, dtype=BF16)
    p.append([lens])
    p.check_attention([1])
    p.check_attention([min(lens, 9)])
    p.check_attention([lens])


def test_rows_that_see_nothing_are_zero():
    p = Paged(n_seqs=3, seed=51, rot=128)
    p.append([2, 0, 40])
    # five rows over two tokens: the first three see none; a sequence of length zero with rows; an ordinary one
    p.check_attention([5, 3, 2], lens=[2, 0, 40])
    p.check_attention([20, 40, 2], lens=[2, 0, 40])
    p.check_attention([5, 3, 2], lens=[2, 0, 40], causal=False)
    assert int(p.cache.status[0]) == 0


def test_one_dominating_token_and_many_small_ones():
    """A key far above the rest, and values that only the many small probabilities carry: they add up."""
    p = Paged(n_seqs=1, Hq=1, H=1, D=64, G=64, W=0, P=64, max_len=4096, reorder=False, outliers=False)
    T = 4096
    k = torch.randn(T, 1, 64, generator=p.g).half() * 0.01
    v = torch.ones(T, 1, 64).half()
    q = torch.ones(1, 1, 64).half()
    k[100], v[100] = 0.2, -1.0
    b = p.batch([T], [T])
    p.cache.append(b, k.cuda(), v.cuda())
    p.ref.append(0, k, v)
    for scale in (0.5, 1.0):
        p.check_attention([1], sm_scale=scale, q=q)


def test_taking_tokens_back():
    """Drafted tokens that were refused: with a ring longer than the window, lens is lowered and the next append goes on."""
    p = Paged(n_seqs=2, seed=61, W=32, R=40, rot=64)
    p.append([100, 50])
    for _ in range(3):
        p.append([8, 5])
        p.check_attention([8, 5])
        for b in range(2):
            p.ref.truncate(b, len(p.ref.rows[b]) - 4)
        p.check_attention([1, 1])


def test_a_shared_prefix():
    p = Paged(n_seqs=2, W=0, P=32, seed=71)
    p.append([96, 0])
    p.page_table[1, :3] = p.page_table[0, :3]
    p.ref.rows[1] = list(p.ref.rows[0])
    p.append([10, 20])
    p.check_attention([10, 20])


def test_a_serving_run_matches_at_every_step():
    """Prompts in chunks beside decoding sequences, rotated keys, mixed lengths: append and attention step by step."""
    p = Paged(n_seqs=3, Hq=6, H=2, D=128, G=32, W=48, R=64, P=32, rot=64, inter=True, dtype=BF16, seed=81)
    r = random.Random(1)
    for new in ([64, 1, 0], [64, 1, 40], [20, 1, 1], [1, 1, 1], [1, 3, 1], [1, 1, 130], [4, 4, 4]):
        p.append(new, pad=r.randint(0, 2))
        p.check_attention(new, pad=r.randint(0, 2), n_splits=r.randint(0, 3))
    p.check_rows()


def test_strided_rows_of_a_packed_projection():
    p = Paged(n_seqs=2, Hq=4, H=2, D=64, G=32, W=16, seed=91, rot=64)
    T = 70
    qkv = (torch.randn(T, 8, 64, generator=p.g) * 2).half()
    dev = qkv.cuda()
    b = p.batch([30, 40], [30, 40])
    p.cache.append(b, dev[:, 4:6], dev[:, 6:8], rope=p.rope)
    p.ref.append(0, qkv[:30, 4:6], qkv[:30, 6:])
    p.ref.append(1, qkv[30:, 4:6], qkv[30:, 6:])
    p.check_rows()
    flat = p.check_attention([30, 40], q=qkv[:, :4].contiguous())
    wide = torch.zeros(T, 8, 64, dtype=F16, device="cuda")
    p.cache.attention(b, dev[:, :4], 1 / 8.0, out=wide[:, 2:6], rope=p.rope)
    assert torch.equal(wide[:, 2:6], flat) and (wide[:, :2] == 0).all() and (wide[:, 6:] == 0).all()
    k, v = torch.zeros(T, 5, 64, dtype=F16, device="cuda"), torch.zeros(T, 2, 64, dtype=F16, device="cuda")
    p.cache.read(b, k[:, 1:3], v)
    assert (k[:, 0] == 0).all() and (k[:, 3:] == 0).all() and k[:, 1:3].abs().sum() > 0


def test_bad_batches_are_skipped_and_reported():
    p = Paged(n_seqs=4, seed=101, rot=128, max_len=200)
    p.append([40, 41, 42, 43])

    def one(lens, starts, status, T=12, max_new=4, max_len=200, slots=None):
        p.cache.status.zero_()
        before = [getattr(p.cache, n).clone() for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")]
        b = p.cache.batch(p.page_table, torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.tensor(starts, dtype=torch.int32, device="cuda"),
                          T, max_new, max_len, None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda"))
        q = torch.randn(T, 4, 128, generator=p.g).half().cuda()
        out = torch.full((T, 4, 128), 9.0, dtype=F16, device="cuda")
        p.cache.attention(b, q, 0.1, out=out, rope=p.rope)
        assert int(p.cache.status[0]) == status
        p.cache.status.zero_()
        k, v = (torch.full((T, 2, 128), 9.0, dtype=F16, device="cuda") for _ in range(2))
        p.cache.read(b, k, v)
        p.cache.append(b, q[:, :2].contiguous(), q[:, 2:].contiguous(), rope=p.rope)
        return out, k, [torch.equal(x.view(torch.uint8), getattr(p.cache, n).view(torch.uint8)) for x, n in zip(before, ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win"))]

    bad = B.SKVQ_STATUS_BAD_BATCH
    # sequences 0 and 3 are fine and have no new rows; sequence 1 is broken in turn
    for lens, starts, extra in (
            ([40, 41, 42, 43], [0, 0, 5, 5, 5], {}),                       # more rows than max_new
            ([40, 201, 42, 43], [0, 0, 1, 1, 1], {}),                      # longer than max_len (and than the page table)
            ([40, -1, 42, 43], [0, 0, 1, 1, 1], {}),
            ([40, 41, 42, 43], [0, 0, 13, 13, 13], dict(max_new=20)),      # rows behind the last
            ([40, 41, 42, 43], [0, 0, -3, 0, 0], {}),
            ([40, 41, 42, 43], [0, 3, 0, 0, 0], {}),
            ([40, 41, 42, 43], [0, 0, 2, 2, 2], dict(slots=[0, 4, 2, 3])),
            ([40, 41, 42, 43], [0, 0, 2, 2, 2], dict(slots=[0, -1, 2, 3]))):
        out, k, same = one(lens, starts, bad, **extra)
        first = 3 if starts == [0, 3, 0, 0, 0] else 0      # there sequence 0 has three rows, its successor's rows run backwards
        assert (out[:first] != 9).any(-1).all() and (out[first:] == 9).all() and (k[first:] == 9).all(), (lens, starts)
        assert all(same) or first, (lens, starts)


def test_bad_pages_are_left_out_and_reported():
    p = Paged(n_seqs=1, W=0, P=16, seed=111, max_len=128)
    p.append([100])
    good = p.page_table.clone()
    for entry in (-1, p.cache.cfg.n_pages, 2 ** 31 - 1, -2 ** 31):
        p.page_table.copy_(good)
        p.page_table[0, 2] = entry           # tokens 32..47
        for new in (1, 100):
            p.cache.status.zero_()
            q = torch.randn(new, 4, 128, generator=p.g).half()
            out = p.cache.attention(p.batch([new], [100]), q.cuda(), 0.1, causal=False)
            assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_PAGE
            without = ref.Reference(1, 4, 2, 128, 64, 0, F16, p.ref.rk, p.ref.rv, p.ref.ak, p.ref.av)
            without.rows[0] = p.ref.rows[0][:32] + p.ref.rows[0][48:]
            for i in (0, new - 1):
                want, _, err, _ = without.attention(0, q[i:i + 1], 0.1, causal=False)
                assert ((out.cpu().double()[i:i + 1] - want).abs() <= err).all()
        p.cache.status.zero_()
        before = p.cache.k_codes.clone()
        k, v = p.keys(100)
        b = p.batch([100], [100])
        got, _ = p.cache.read(b, torch.full((100, 2, 128), 9.0, dtype=F16, device="cuda"))
        assert (got[32:48] == 9).all() and int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_PAGE
        p.cache.status.zero_()
        p.cache.append(b, k.cuda(), v.cuda())
        assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_PAGE
        held = int(good[0, 2])
        assert torch.equal(p.cache.k_codes[held], before[held])
        p.ref.rows[0] = []
        p.ref.append(0, k, v)                # the tokens of the bad page are not compared: their page still holds the older rows
        p.page_table.copy_(good)
        codes = p.cache.k_codes.cpu()
        for t in (0, 31, 48, 99):
            row = p.ref.rows[0][t]
            assert torch.equal(codes[int(good[0, t // 16]), :, t % 16], row[2][:, 0::2] | row[2][:, 1::2] << 4)
        p.cache.append(p.batch([100], [100]), k.cuda(), v.cuda())


def test_pages_beyond_32_bits():
    """Page numbers whose rows lie past 2^32 bytes of the pool."""
    p = Paged(n_seqs=1, Hq=8, H=8, D=128, G=64, W=16, P=256, max_len=300, spare=34000, seed=121)
    assert p.cache.k_codes.numel() > 2 ** 32 and int(p.page_table.min()) >= 34000
    p.append([280])
    p.check_attention([1])
    p.check_attention([40])
    pt = p.page_table.cpu().long()
    for t in (0, 255, 256, 279):
        row = p.ref.rows[0][t]
        assert torch.equal(p.cache.k_codes[pt[0, t // 256], :, t % 256].cpu(), row[2][:, 0::2] | row[2][:, 1::2] << 4)


def test_capture_replay_streams_and_shared_calls():
    """A decode step captured into two graphs and replayed with new inputs, beside calls on another stream."""
    p = Paged(n_seqs=2, seed=131, rot=128, W=16)
    p.append([100, 60])
    q = [torch.randn(2, 4, 128, generator=p.g).half() for _ in range(3)]
    qd, lens = q[0].cuda(), torch.tensor([101, 61], dtype=torch.int32, device="cuda")
    k, v = p.keys(2)
    kd, vd = k.cuda(), v.cuda()
    b = p.cache.batch(p.page_table, lens, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), 2, 1, 200)
    outs = [torch.zeros(2, 4, 128, dtype=F16, device="cuda") for _ in range(2)]
    graphs = []
    side = torch.cuda.Stream()
    for out in outs:
        side.wait_stream(torch.cuda.current_stream())
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            p.cache.append(b, kd, vd, rope=p.rope)
            p.cache.attention(b, qd, 0.1, out=out, rope=p.rope)
        graphs.append(gr)
    for i in range(2):
        p.ref.append(i, k[i:i + 1], v[i:i + 1])
    for step in range(1, 3):
        qd.copy_(q[step])
        torch.cuda.synchronize()
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        with torch.cuda.stream(s1):
            graphs[0].replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s2):                       # the second graph beside an eager call on another stream
            graphs[1].replay()
        other = p.cache.attention(b, qd, 0.1, rope=p.rope, stream=s1)
        torch.cuda.synchronize()
        for i in range(2):
            want, _, err, _ = p.ref.attention(i, q[step][i:i + 1], 0.1)
            for o in (*outs, other):
                assert ((o.cpu().double()[i:i + 1] - want).abs() <= err).all()
        # the next step: one more token each, lengths changed on the device
        k, v = p.keys(2)
        kd.copy_(k)
        vd.copy_(v)
        lens += 1
        for i in range(2):
            p.ref.append(i, k[i:i + 1], v[i:i + 1])
    p.cache.append(b, kd, vd, rope=p.rope)
    p.check_rows()


def test_results_repeat_bit_for_bit():
    p = Paged(n_seqs=3, seed=141, W=32)
    p.append([390, 17, 201])
    for new in ([1, 1, 1], [60, 17, 130]):
        q = torch.randn(sum(new), 4, 128, generator=p.g).half().cuda()
        b = p.batch(new, p.lens())
        first = p.cache.attention(b, q, 0.1)
        for _ in range(5):
            assert torch.equal(p.cache.attention(b, q, 0.1), first)


def test_many_sequences():
    n = 300
    p = Paged(n_seqs=n, Hq=2, H=1, D=64, G=64, W=8, P=16, seed=151, max_len=48)
    r = random.Random(2)
    p.append([r.randint(0, 40) for _ in range(n)])
    p.append([r.randint(0, 1) for _ in range(n)])
    p.check_attention([min(1, L) for L in p.lens()])


def test_prompts_of_one_and_two_row_blocks_in_turn():
    """Items of fewer than 128 packed rows beside items of more, many tiles of both for every CTA: the second row block is idle for
    several tiles and has to stay in step.  (One that ran ahead waited on a barrier two phases behind and got through at once.)"""
    p = Paged(n_seqs=8, Hq=32, H=32, D=64, G=32, W=16, P=64, seed=161, max_len=1300, dtype=BF16, outliers=False)
    p.append([1100, 1200] * 4)
    new = [100, 200, 40, 129, 128, 300, 60, 140]
    q = torch.randn(sum(new), 32, 64, generator=p.g).to(BF16)
    b = p.batch(new, p.lens())
    out = p.cache.attention(b, q.cuda(), 0.125)
    assert int(p.cache.status[0]) == 0
    got, at = out.cpu().double(), 0
    for i, n in enumerate(new):
        rows = sorted({0, 1, n // 2, n - 1})
        for r in rows:      # a row and all behind it taken away: the same tokens seen
            L = len(p.ref.rows[i])
            K, V = p.ref.values(i, "k"), p.ref.values(i, "v")
            off = p.ref.score_error(i)
            lim = L - n + r + 1
            for h in (0, 13, 31):
                qr = q[at + r, h].double()[p.ref.rk[h]]
                s = 0.125 * (K[:lim, h] @ qr)
                w = torch.softmax(s, 0)
                o = w @ V[:lim, h]
                ds = 0.125 * float((off[:lim, h] @ qr.abs()).max())
                err = (w @ V[:lim, h].abs()) * (2.0 ** -10 + 2 * ds + 2.0 ** -21 + lim * 2.0 ** -23)
                err = err + o.abs() * 2.0 ** -8 * 1.01 + 1e-7
                assert ((got[at + r, h][p.ref.rv[h]] - o).abs() <= err).all(), (i, r, h)
        at += n


@pytest.mark.parametrize("lens,new,kw", [
    ([20000], [1], dict(Hq=4, H=1, D=128, G=64, W=128, P=64)),                        # one item: more partial results than a warp has lanes
    ([4100, 900, 0, 2500], [1, 1, 0, 1], dict(Hq=4, H=2, D=64, G=32, W=40, P=16, dtype=BF16)),      # equal pieces of every item, some of them empty
    ([5000, 33], [4, 1], dict(Hq=8, H=2, D=128, G=128, W=0, P=256)),                  # the same, two tiles of rows
    ([1800, 1700, 40, 1601, 1, 1650, 1700, 1900], [1] * 8, dict(Hq=32, H=32, D=64, G=64, W=16, P=64)),      # equal shares of the step
    ([1800, 1700, 40, 1601, 1, 1650, 1700, 1900], [3, 1, 2, 4, 1, 4, 0, 2], dict(Hq=48, H=16, D=64, G=64, W=16, P=64)),      # the same, two tiles of rows
])
def test_long_contexts_however_the_step_is_cut(lens, new, kw):
    p = Paged(n_seqs=len(lens), seed=171, max_len=max(lens), **kw)
    p.append(lens)
    p.check_attention(new)
    p.check_attention(new, max_len=max(lens) + 5000 if max(lens) + 5000 <= p.max_pages * p.P else p.max_pages * p.P)      # a loose bound of the longest
    assert int(p.cache.status[0]) == 0


@pytest.mark.parametrize("new,n_splits", [([1, 1], 0), ([1, 1], 3), ([4, 3], 0), ([20, 150], 0), ([0, 300], 0)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_query_that_is_not_a_number_spoils_its_own_row_alone(new, n_splits, dtype):
    p = Paged(n_seqs=2, Hq=8, H=2, D=128, G=64, W=32, P=64, seed=181, max_len=2000, dtype=dtype)
    p.append([400, 1900])
    T = sum(new)
    q = torch.randn(T, 8, 128, generator=p.g).to(dtype)
    b = p.batch(new, p.lens())
    lse = torch.empty(T, 8, device="cuda")
    good = p.cache.attention(b, q.cuda(), 0.1, n_splits=n_splits, lse=lse)
    bad = q.clone()
    bad[0, 3, 5] = bad[T - 1, 6] = math.nan
    lse2 = torch.empty(T, 8, device="cuda")
    out = p.cache.attention(b, bad.cuda(), 0.1, n_splits=n_splits, lse=lse2)
    spoilt = torch.zeros(T, 8, dtype=torch.bool, device="cuda")
    spoilt[0, 3] = spoilt[T - 1, 6] = True
    assert torch.isnan(out[spoilt]).all() and torch.isnan(lse2[spoilt]).all()
    assert torch.equal(out[~spoilt], good[~spoilt]) and torch.equal(lse2[~spoilt], lse[~spoilt])
