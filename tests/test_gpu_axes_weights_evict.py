"""Rotations with several axes, accumulated attention weights and eviction on the GPU against plain forms (shrink_reference).

Rotations, kept tokens and moved rows bit for bit; weights against 64 bits with the error that shrink_reference.weights counts."""
import math

import pytest
import torch

import paged_reference as ref
import shrink_reference as plain
import test_gpu_rope_paged as base
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build
from test_gpu_paged_guards import GuardedPaged, guarded

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
bits, gen = base.bits, base.gen


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


# ------------------------------------------------------------------------------------------------ rotations with several axes
def assignment(pairs, n_axes, how, g):
    if how == "runs":
        return sorted(int(a) for a in torch.randint(0, n_axes, (pairs,), generator=g))
    if how == "turns":
        return [j % n_axes for j in range(pairs)]
    return [int(a) for a in torch.randint(0, n_axes, (pairs,), generator=g)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("T,Hq,Hk,D,rot,inter,n_axes,how", [
    (1, 1, 0, 2, 2, False, 1, "runs"), (3, 4, 1, 128, 128, False, 3, "runs"), (67, 32, 8, 128, 128, True, 3, "turns"), (130, 5, 5, 64, 32, False, 2, "any"),
    (33, 3, 2, 80, 48, True, 4, "any"), (1000, 8, 2, 128, 64, True, 2, "runs"), (19, 2, 1, 96, 20, False, 4, "turns"), (7, 3, 3, 33, 30, True, 3, "any"),
    (5, 2, 2, 512, 256, False, 4, "any"), (260, 6, 2, 64, 16, False, 3, "runs"), (4100, 4, 4, 64, 64, False, 3, "runs"),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_axes_bit_exact(dtype, T, Hq, Hk, D, rot, inter, n_axes, how, inverse):
    g = gen(T * 7 + D)
    of_pair = assignment(rot // 2, n_axes, how, g)
    axes = B.RopeAxes(of_pair)
    qkv = torch.randn(T, Hq + Hk + 1, D, generator=g).to(dtype)
    table = ref.table64(rot, 500).float()
    pos = torch.randint(0, 500, (axes.n_axes, T), generator=g, dtype=torch.int32)
    rope = B.RopeTable(table.cuda(), rot, inter)
    dev = qkv.cuda()
    q, k = dev[:, :Hq], dev[:, Hq:Hq + Hk] if Hk else None
    q_out = torch.full((T, Hq, D), 3.0, dtype=dtype, device="cuda")
    k_out = torch.full((T, Hk, D), 3.0, dtype=dtype, device="cuda") if Hk else None
    rope.apply_axes(axes, pos.cuda(), q, q_out, k, k_out, inverse=inverse)
    cs = plain.axis_angles(table, pos, of_pair)
    want = ref.rotate32(qkv, cs, rot, inter, inverse)
    assert torch.equal(bits(q_out.cpu()), bits(want[:, :Hq]))
    if Hk:
        assert torch.equal(bits(k_out.cpu()), bits(want[:, Hq:Hq + Hk]))
    assert torch.equal(bits(dev.cpu()), bits(qkv))
    exact = ref.rotate(qkv[:, :Hq], cs, rot, inter, inverse)      # 64 bits: three roundings of 2^-24 of the terms, one of the type
    terms = qkv[:, :Hq].double().abs().amax(-1, keepdim=True) * 2
    assert ((q_out.cpu().double() - exact).abs() <= terms * 2.0 ** -23 + exact.abs() * torch.finfo(dtype).eps / 2 * 1.01 + 2.0 ** -25).all()
    rope.apply_axes(axes, pos.t().contiguous().cuda().t(), q, None, k, None, inverse=inverse)      # positions [T, n_axes]; in place
    assert torch.equal(bits(dev.cpu()[:, :Hq + Hk]), bits(want[:, :Hq + Hk])) and torch.equal(bits(dev.cpu()[:, -1]), bits(qkv[:, -1]))


def test_one_axis_and_equal_positions_are_the_plain_rotation():
    g = gen(3)
    x = torch.randn(300, 5, 128, generator=g).half().cuda()
    rope = B.RopeTable.build(128, 4000)
    pos = torch.randint(0, 4000, (300,), generator=g, dtype=torch.int32).cuda()
    want, a, b = (torch.empty_like(x) for _ in range(3))
    rope.apply(pos, x, want)
    rope.apply_axes(B.RopeAxes([0] * 64), pos[None], x, a)
    rope.apply_axes(B.RopeAxes.runs([16, 24, 24]), pos[None].expand(3, -1), x, b)      # an axis stride of 0
    assert torch.equal(bits(a), bits(want)) and torch.equal(bits(b), bits(want))


def test_axes_gradient_by_formula_and_by_differences():
    T, H, D, rot, of_pair = 9, 3, 64, 48, [0] * 5 + [1] * 9 + [2] * 10
    g = gen(5)
    x, dy = torch.randn(T, H, D, generator=g), torch.randn(T, H, D, generator=g)
    table = ref.table64(rot, 40).float()
    pos = torch.randint(0, 40, (3, T), generator=g, dtype=torch.int32)
    rope, axes = B.RopeTable(table.cuda(), rot, True), B.RopeAxes(of_pair)
    dx = torch.empty(T, H, D, device="cuda")
    rope.apply_axes(axes, pos.cuda(), dy.cuda(), dx, inverse=True)
    x64 = x.double().requires_grad_()
    cs = plain.axis_angles(table, pos, of_pair)[:, None].double()
    x1, x2, c, s = x64[..., 0:rot:2], x64[..., 1:rot:2], cs[..., 0], cs[..., 1]
    y = torch.cat((torch.stack((x1 * c - x2 * s, x1 * s + x2 * c), -1).flatten(-2), x64[..., rot:]), -1)
    (y * dy.double()).sum().backward()
    assert (dx.cpu().double() - x64.grad).abs().max() <= 4 * float(dy.abs().max()) * 2.0 ** -24
    for seed in range(4):      # the rotation is linear: one step is exact but for roundings
        d = torch.randn(T, H, D, generator=gen(seed))
        out = [torch.empty(T, H, D, device="cuda") for _ in range(2)]
        rope.apply_axes(axes, pos.cuda(), (x + d).cuda(), out[0])
        rope.apply_axes(axes, pos.cuda(), (x - d).cuda(), out[1])
        diff = float((((out[0] - out[1]).cpu().double() / 2) * dy.double()).sum())
        assert abs(diff - float((dx.cpu().double() * d.double()).sum())) <= T * H * D * 10 * float(dy.abs().max()) * 2.0 ** -22


def test_a_position_outside_the_table_on_any_axis_leaves_the_token():
    table = ref.table64(64, 10).float()
    rope, axes = B.RopeTable(table.cuda(), 64), B.RopeAxes.runs([10, 12, 10])
    x = torch.randn(5, 2, 64).half()
    pos = torch.tensor([[0, 10, 3, 3, 9], [1, 1, -1, 3, 9], [2, 2, 2, 2**31 - 1, 9]], dtype=torch.int32)
    out, status = torch.full((5, 2, 64), 5.0, dtype=F16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    rope.apply_axes(axes, pos.cuda(), x.cuda(), out, status=status)
    assert int(status.item()) == B.SKVQ_STATUS_BAD_POSITION and (out.cpu()[1:4] == 5).all()
    want = ref.rotate32(x, plain.axis_angles(table, pos.clamp(0, 9), [0] * 10 + [1] * 12 + [2] * 10), 64, False)
    assert torch.equal(out.cpu()[[0, 4]], want[[0, 4]])


# ------------------------------------------------------------------------------------------------ accumulated weights
class Weighed(base.Paged):
    """A cache, its plain reference and a weight tensor whose unused entries are marked."""

    def __init__(self, capacity=401, **kw):
        super().__init__(**kw)
        self.capacity, self.guards = capacity, {}
        f = self.cache.cfg
        self.weights = guarded(torch.full((f.n_slots, f.n_kv_heads, capacity), 7.0, device="cuda"), self.guards, "weights")
        self.workspace_guards = []

    def slot(self, b):
        return b if self.slots is None else int(self.slots[b])

    def lse(self, new, q, sm_scale, causal):
        """The rows' log-sum-exp from 64 bits."""
        out, at = torch.zeros(q.shape[0], self.Hq), 0
        for b, n in enumerate(new):
            out[at:at + n] = self.ref.attention(b, q[at:at + n], sm_scale, causal)[1].float()
            at += n
        return out

    def check(self, new, causal=True, last=0, pad=0, sm_scale=None, q=None, lse=None, old=None, max_new=None, out=None):
        """One call on weights that hold `old` (random by default), new tokens' entries not a number; its result against the plain form."""
        sm_scale = 1 / math.sqrt(self.D) if sm_scale is None else sm_scale
        T, lens, f = sum(new), self.lens(), self.cache.cfg
        q = torch.randn(T + pad, self.Hq, self.D, generator=self.g).to(self.dtype) if q is None else q
        lse = torch.cat((self.lse(new, q[:T], sm_scale, causal), torch.full((pad, self.Hq), math.nan))) if lse is None else lse
        before = torch.rand(f.n_slots, f.n_kv_heads, self.capacity, generator=self.g) if old is None else old.clone()
        for b, (n, L) in enumerate(zip(new, lens)):
            before[self.slot(b), :, max(L - n, 0):L] = math.nan
        source = before.cuda()
        target = self.weights if out is None else source
        if out is None:
            target.fill_(7.0)
        batch = self.batch(new, lens, pad, max_new)
        size = B.skvq_paged_weights_workspace_size(f, batch, last)
        ws = guarded(torch.full((max(size, 16),), 0xFF, dtype=torch.uint8, device="cuda"), self.guards, "workspace")
        self.cache.accumulate_weights(batch, q.cuda(), lse.cuda(), source, sm_scale, out=target, causal=causal, rope=self.rope, last=last, workspace=ws[:size] if size else ws)
        torch.cuda.synchronize()
        for name, g in self.guards.items():
            assert g.margins_intact(), f"bytes next to {name} were overwritten"
        got, at = target.cpu(), 0
        used = torch.zeros(f.n_slots, self.capacity, dtype=torch.bool)
        for b, (n, L) in enumerate(zip(new, lens)):
            want, err = plain.weights(self.ref, b, q[at:at + n], lse[at:at + n], before[self.slot(b)], sm_scale, causal, last)
            off = (got[self.slot(b), :, :L].double() - want).abs() - err
            assert not torch.isnan(got[self.slot(b), :, :L]).any() and (off <= 0).all(), (b, n, L, float(off.max()) if L else 0.0)
            used[self.slot(b), :L] = True
            at += n
        rest = ~used[:, None].expand_as(got)
        assert (got[rest] == 7).all() if out is None else torch.equal(got[rest], before[rest])
        return got


@pytest.mark.parametrize("kw", base.SHAPES)
def test_weights_of_single_tokens(kw):
    p = Weighed(n_seqs=4, seed=21, slots=[4, 0, 2, 1], **kw)
    p.append([1, 300, 33, 0])
    p.check([1, 1, 1, 0])
    p.append([1, 1, 1, 1])
    p.check([1, 1, 1, 1])
    p.check([1, 1, 0, 1], out="same")
    assert int(p.cache.status[0]) == 0


@pytest.mark.parametrize("kw", base.SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_several_rows(kw, causal):
    p = Weighed(n_seqs=4, seed=31, **kw)
    p.append([70, 129, 5, 200])
    p.check([4, 7, 5, 1], causal=causal, pad=2)
    p.append([3, 2, 16, 17])
    p.check([3, 2, 16, 17], causal=causal)
    p.check([0, 0, 21, 0], causal=causal)
    p.check([3, 2, 16, 17], causal=causal, last=2)
    p.check([3, 2, 16, 17], causal=causal, last=1, max_new=40)


@pytest.mark.parametrize("kw", base.SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_prompts_and_chunks(kw, causal):
    p = Weighed(n_seqs=3, seed=41, **kw)
    p.append([150, 1, 77])
    p.check([150, 1, 77], causal=causal, pad=5)
    p.append([130, 200, 64])
    p.check([130, 200, 64], causal=causal)
    p.check([130, 200, 64], causal=causal, last=40)


@pytest.mark.parametrize("lens", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_weights_around_every_boundary(lens):
    p = Weighed(n_seqs=1, Hq=2, H=1, D=64, G=32, W=16, P=16, seed=lens, dtype=BF16, capacity=400)
    p.append([lens])
    p.check([1])
    p.check([min(lens, 9)])
    p.check([lens])


def test_rows_that_add_nothing():
    p = Weighed(n_seqs=3, seed=51, rot=128)
    p.append([2, 0, 40])
    # more rows than tokens: the first see none; rows of an empty sequence; then rows whose lse or query is not finite
    for new in ([5, 3, 2], [20, 40, 2]):
        q = torch.randn(sum(new), p.Hq, p.D, generator=p.g).to(p.dtype)
        lse = torch.randn(sum(new), p.Hq, generator=p.g) + 3
        got = p.check(new, q=q, lse=lse)
        assert (got[0, :, :2] > 0).all()
        p.check(new, q=q, lse=lse, causal=False)
    new = [2, 0, 30]
    for at in range(4):
        q = torch.randn(32, p.Hq, p.D, generator=p.g).to(p.dtype)
        lse = torch.randn(32, p.Hq, generator=p.g) + 3
        lse[3 * at, 1], lse[5 + at, 0], lse[9 + at, 2] = math.nan, math.inf, -math.inf
        q[20, at, 5], q[21, at, 127], q[0, at, 0] = math.inf, math.nan, -math.inf
        p.check(new, q=q, lse=lse)
    nothing = torch.full((32, p.Hq), -math.inf)
    old = torch.rand(3, p.H, p.capacity, generator=p.g)
    got = p.check(new, lse=nothing, old=old)
    assert torch.equal(got[2, :, :10], old[2, :, :10]) and (got[2, :, 10:40] == 0).all()
    assert int(p.cache.status[0]) == 0


@pytest.mark.parametrize("rows", [1, 40])
def test_weights_without_old_ones_and_scales(rows):
    p = Weighed(n_seqs=2, seed=61, Hq=8, H=2, G=32, dtype=BF16)
    p.append([200, 90])
    q = torch.randn(2 * rows, p.Hq, p.D, generator=p.g).to(p.dtype)
    for scale in (0.0, -0.05, 0.02):
        p.check([rows, rows], q=q, sm_scale=scale)
    for size in (1e-6, 300.0):      # queries at the ends of what fp16 resolves; scores stay small
        p.check([rows, rows], q=(q.float() * size).to(BF16), sm_scale=0.02 / size)
    lse = p.lse([rows, rows], q, 0.1, True)
    lens, batch = p.lens(), p.batch([rows, rows], p.lens())
    a, b = torch.full((2, 2, p.capacity), 7.0, device="cuda"), torch.full((2, 2, p.capacity), 7.0, device="cuda")
    p.cache.accumulate_weights(batch, q.cuda(), lse.cuda(), torch.zeros_like(a), 0.1, out=a, rope=p.rope)
    p.cache.accumulate_weights(batch, q.cuda(), lse.cuda(), None, 0.1, out=b, rope=p.rope)
    assert torch.equal(a, b) and (a[0, :, lens[0]:] == 7).all()


def test_sequences_without_new_tokens_are_copied():
    p = Weighed(n_seqs=2, seed=62)
    p.append([300, 20])
    p.check([0, 0], max_new=0)
    p.check([0, 0], max_new=3)
    p.check([0, 1])


def test_weights_skip_bad_sequences_and_bad_pages():
    for rows in (1, 40):
        p = Weighed(n_seqs=4, seed=71, P=16, W=16, slots=[0, 1, 2, 3])
        p.append([100, 100, 100, 100])
        q = torch.randn(4 * rows, p.Hq, p.D, generator=p.g).to(p.dtype).cuda()
        lse = torch.full((4 * rows, p.Hq), 4.0, device="cuda")
        good, bad = (torch.full((4, p.H, 401), 7.0, device="cuda") for _ in range(2))
        p.cache.accumulate_weights(p.batch([rows] * 4, p.lens()), q, lse, None, 0.1, out=good)
        assert int(p.cache.status[0]) == 0
        b = p.batch([rows] * 4, [100, 500, 100, 100], max_len=400)      # longer than max_len
        p.slots[2] = 9                                               # no such slot
        p.page_table[0, 3], p.page_table[3, 6] = -1, 10 ** 6         # tokens 48..63; tokens 96..111, inside the window
        p.cache.accumulate_weights(b, q, lse, None, 0.1, out=bad)
        assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_BATCH | B.SKVQ_STATUS_BAD_PAGE
        assert (bad[1:3] == 7).all()
        assert torch.equal(bad[0, :, :48], good[0, :, :48]) and torch.equal(bad[0, :, 64:], good[0, :, 64:]) and (bad[0, :, 48:64] == 0).all()
        assert torch.equal(bad[3, :, :96], good[3, :, :96]) and (bad[3, :, 96:100] == 0).all() and (bad[3, :, 100:] == 7).all()
        no_window = B.SkvqPagedCache(p.Hq, p.H, p.D, 64, 0, 16, p.cache.cfg.n_pages, 4, device="cuda")
        p.slots[2], p.slots[1] = -1, 4
        b = no_window.batch(p.page_table, b.keep[1], b.keep[2], b.n_tokens, rows, 400, slots=p.slots)
        bad.fill_(7)
        no_window.accumulate_weights(b, q, lse, None, 0.1, out=bad)      # slots matter without a window too
        assert int(no_window.status[0]) == B.SKVQ_STATUS_BAD_BATCH | B.SKVQ_STATUS_BAD_PAGE and (bad[1:3] == 7).all()


def test_weights_of_a_long_context_are_attentions_own():
    """Many tokens, few and many rows: the sum over tokens of what a row gives is 1, and runs agree bit for bit."""
    H, Hq, D, L, P = 2, 8, 128, 70001, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    n_pages = -(-L // P)
    cache = B.SkvqPagedCache(Hq, H, D, 32, 128, P, n_pages, 1, BF16)
    table = torch.randperm(n_pages, generator=g, device="cuda").int()[None]
    lens, k = torch.tensor([L], dtype=torch.int32, device="cuda"), torch.randn(L, H, D, generator=g, device="cuda").to(BF16)
    cache.append(cache.batch(table, lens, torch.tensor([0, L], dtype=torch.int32, device="cuda"), L, L, L), k, k)
    for rows in (1, 3, 65, 300):
        batch = cache.batch(table, lens, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), rows, rows, L)
        q, lse = torch.randn(rows, Hq, D, generator=g, device="cuda").to(BF16), torch.empty(rows, Hq, device="cuda")
        cache.attention(batch, q, D ** -0.5, lse=lse)
        a, b = cache.new_weights(L + 3), cache.new_weights(L + 3)
        cache.accumulate_weights(batch, q, lse, None, D ** -0.5, out=a)
        cache.accumulate_weights(batch, q, lse, None, D ** -0.5, out=b)
        assert torch.equal(a, b) and (a[..., L:] == 0).all()
        # attention rounds keys and queries' products to fp16: 2^-11 of scores up to 20
        total = a.double().sum(-1)[0]
        assert (total / (rows * Hq // H) - 1).abs().max() <= 20 * 2.0 ** -10, total


@pytest.mark.parametrize("n", [129, 700, 2048])
def test_weights_of_very_many_sequences(n):
    """Ragged batches up to the largest: every sequence as a call of its own gives it -- bit for bit where few rows are counted (a token's
    sum does not depend on the cut), to fp32's sums where many are."""
    H, Hq, D, P, g = 2, 4, 64, 16, torch.Generator(device="cuda").manual_seed(n)
    cpu = gen(n)
    lens = torch.randint(0, 90, (n,), generator=cpu)
    lens[5], lens[n - 1], lens[7] = 900, 333, 0
    new = torch.minimum(torch.randint(0, 4, (n,), generator=cpu), lens)
    new[n // 2] = lens[n // 2] = 64      # one of many rows
    new[n - 1] = 50
    pages = -(-900 // P)
    cache = B.SkvqPagedCache(Hq, H, D, 32, 8, P, 4096, n, F16)
    for name in ("k_codes", "v_codes"):
        getattr(cache, name).copy_(torch.randint(0, 256, cache.k_codes.shape, generator=g, device="cuda", dtype=torch.uint8))
    for name in ("k_meta", "v_meta", "k_win", "v_win"):
        getattr(cache, name).copy_(torch.rand(getattr(cache, name).shape, generator=g, device="cuda") * 0.1)
    table = torch.randint(0, 4096, (n, pages), generator=g, device="cuda", dtype=torch.int32)
    starts = torch.cat((torch.zeros(1, dtype=torch.int64), new.cumsum(0)))
    T = int(starts[-1])
    q, lse = torch.randn(T + 1, Hq, D, generator=g, device="cuda").half(), torch.full((T + 1, Hq), 3.0, device="cuda")
    dev = lambda x: x.to(torch.int32).cuda()      # noqa: E731
    all_lens, old = dev(lens), torch.rand(n, H, 901, generator=g, device="cuda")
    got = torch.full_like(old, 7.0)
    cache.accumulate_weights(cache.batch(table, all_lens, dev(starts), T, 64, 900), q, lse, old, 0.1, out=got)
    assert int(cache.status[0]) == 0
    for b in [0, 1, 5, 7, 31, 32, 33, 127, 128, n // 2, n - 2, n - 1]:
        m, L = int(new[b]), int(lens[b])
        one = torch.full_like(old, 7.0)
        # the same bound on new tokens: it chooses how rows lie side by side, and so the order in which a token's rows are added
        batch = cache.batch(table[b:b + 1].contiguous(), all_lens[b:b + 1], dev(torch.tensor([0, m])), max(m, 1), 64, 900, slots=dev(torch.tensor([b])))
        cache.accumulate_weights(batch, q[starts[b]:starts[b] + max(m, 1)], lse[:max(m, 1)], old, 0.1, out=one)
        assert (got[b, :, L:] == 7).all()
        if m * Hq // H <= 16:
            assert torch.equal(got[b, :, :L], one[b, :, :L]), b
        else:
            assert (got[b, :, :L] - one[b, :, :L]).abs().max() <= m * Hq // H * 2.0 ** -22 * float(one[b, :, :L].max()), b
    kept, lens_out, _ = cache.evict(cache.batch(table, all_lens, dev(starts), 0, 0, 900), got.clone(), 20, 2, 8, weights_out=torch.zeros_like(got),
                                    page_table_out=torch.arange(2 * n, device="cuda", dtype=torch.int32).view(n, 2))
    assert torch.equal(lens_out, all_lens.clamp(max=20))
    for b in (0, 5, 7, 128, n - 1):
        mine = [plain.chosen(got[b, h, :int(lens[b])].tolist(), int(lens[b]), 20, 2, 8) for h in range(H)]
        assert kept[b].tolist() == [m + [-1] * (20 - len(m)) for m in mine], b


# ------------------------------------------------------------------------------------------------ eviction
def shrink(ref_cache, b, kept):
    """The plain cache after the move: token i of head h is token kept[h][i]."""
    rows = ref_cache.rows[b]
    n = len(kept[0])
    ref_cache.rows[b] = [tuple(torch.stack([rows[kept[h][i]][part][h] for h in range(ref_cache.H)]) for part in range(6)) for i in range(n)]


def check_rows(p, page_table, slots, lens, ring_from):
    """Codes, parameters and the ring's rows of every sequence bit for bit."""
    c, pt, P = p.cache, page_table.cpu().long(), p.P
    codes, meta, win = [c.k_codes.cpu(), c.v_codes.cpu()], [c.k_meta.cpu(), c.v_meta.cpu()], [c.k_win.cpu(), c.v_win.cpu()]
    for b, rows in enumerate(p.ref.rows):
        assert len(rows) == int(lens[b])
        for t, row in enumerate(rows):
            for s in range(2):
                assert torch.equal(codes[s][pt[b, t // P], :, t % P], row[2 + 2 * s][:, 0::2] | row[2 + 2 * s][:, 1::2] << 4), (b, t, s)
                assert torch.equal(bits(meta[s][pt[b, t // P], :, t % P]), bits(row[3 + 2 * s])), (b, t, s)
                if p.W and t >= int(ring_from[b]):
                    assert torch.equal(bits(win[s][slots[b], :, t % c.cfg.ring_tokens]), bits(row[s])), (b, t, s)


EVICT = [
    dict(keep=60, first=4, recent=40), dict(keep=40, first=0, recent=40), dict(keep=64, first=0, recent=33), dict(keep=129, first=16, recent=64),
    dict(keep=41, first=1, recent=40), dict(keep=300, first=4, recent=250), dict(keep=130, first=4, recent=40),
]


@pytest.mark.parametrize("kw", [dict(D=128, G=64, P=16, W=32, R=37), dict(D=128, G=32, P=32, W=20, R=33, dtype=BF16), dict(D=64, G=32, H=3, Hq=3, P=16, W=16),
                                dict(D=64, G=64, H=1, Hq=1, P=128, W=5, R=64), dict(D=128, G=128, P=64, W=0)])
@pytest.mark.parametrize("args", EVICT)
@pytest.mark.parametrize("where", ["in place", "elsewhere"])
def test_evict_bit_exact(kw, args, where):
    lens = [129, 0, 300, 61, 130, 1]
    p = base.Paged(n_seqs=6, seed=5, max_len=320, spare=6 * 20, slots=[4, 0, 2, 1, 11, 3], **kw)
    p.append(lens)
    p.append([0, 0, 2, 0, 1, 0])
    lens = p.lens()
    c, g = p.cache, gen(args["keep"])
    w = torch.floor(torch.rand(12, p.H, 333, generator=g) * 12) / 4 - 1      # many ties, negative ones too
    w[w == 0] *= -1
    w[2, :, 50:53], w[2, :, 60], w[4, :, 9], w[2, :, 100] = math.nan, math.inf, -math.inf, -0.0
    table_out = slots_out = None
    want_slots, want_table, extra = [4, 0, 2, 1, 11, 3], p.page_table, {}
    if where == "elsewhere":
        need = -(-min(args["keep"], 302) // p.P)
        table_out = torch.randperm(6 * 20, generator=g)[:6 * need].view(6, need).int().cuda()
        want_slots, want_table = [5, 6, 7, 1, 8, 9], table_out
        slots_out = torch.tensor(want_slots, dtype=torch.int32, device="cuda")
        extra = dict(page_table_out=table_out, slots_out=slots_out, weights_out=torch.full_like(w, 7.0).cuda())
    wd = w.cuda()
    batch = p.batch([0] * 6, lens)
    kept, lens_out, ring_from = c.evict(batch, wd, **args, **extra)
    after = extra.get("weights_out", wd).cpu()
    used = torch.zeros(12, 333, dtype=torch.bool)
    for b, L in enumerate(lens):
        mine = [plain.chosen(w[p.slots[b], h].tolist(), L, **args) for h in range(p.H)]
        n = min(L, args["keep"])
        assert kept[b].cpu().tolist() == [m + [-1] * (args["keep"] - n) for m in mine], b
        for h in range(p.H):
            got = after[want_slots[b], h, :n]
            assert torch.equal(got.view(torch.int32), w[p.slots[b], h][mine[h]].view(torch.int32)), (b, h)
        used[want_slots[b], :n] = True
        shrink(p.ref, b, mine)
    rest = ~used[:, None].expand_as(after)
    assert torch.equal(after[rest].view(torch.int32), (w if where == "in place" else torch.full_like(w, 7.0))[rest].view(torch.int32))
    assert lens_out.tolist() == [min(L, args["keep"]) for L in lens]
    R = c.cfg.ring_tokens
    for b, L in enumerate(lens):      # what the ring holds: the recent tokens of a shortened sequence, all it had of a whole one
        assert int(ring_from[b]) == (max(L - (min(R, args["recent"]) if L > args["keep"] else R), 0) - max(L - args["keep"], 0) if p.W else 0)
    check_rows(p, want_table, want_slots, lens_out, ring_from)
    assert int(c.status[0]) == 0


def test_the_batchs_own_lengths_may_be_overwritten():
    p = base.Paged(n_seqs=3, H=8, Hq=8, D=64, G=32, seed=6, R=50)
    p.append([250, 40, 390])
    w = torch.rand(3, 8, 400, generator=gen(1)).cuda()
    first = torch.tensor([0, 0, 345], dtype=torch.int32, device="cuda")
    lens = torch.tensor(p.lens(), dtype=torch.int32, device="cuda")
    batch = p.cache.batch(p.page_table, lens, torch.zeros(4, dtype=torch.int32, device="cuda"), 0, 0, 390, ring_from=first)
    kept, lens_out, ring_from = p.cache.evict(batch, w, 100, 4, 60, lens_out=lens, ring_from_out=first)
    assert lens_out is lens and lens.tolist() == [100, 40, 100]
    # the ring holds 50 tokens: 200..249 shift by 150; the last begins at 345 and shifts by 290
    assert ring_from.tolist() == [50, 0, 55]
    kept = kept.cpu()
    for b in range(3):
        shrink(p.ref, b, [[t for t in kept[b, h].tolist() if t >= 0] for h in range(8)])
    check_rows(p, p.page_table, [0, 1, 2], lens, ring_from)


def test_evict_skips_bad_sequences_and_bad_pages():
    p = base.Paged(n_seqs=4, seed=7, slots=[0, 1, 2, 3], P=16)
    p.append([100, 100, 100, 100])
    before = [getattr(p.cache, n).clone() for n in ("k_codes", "v_codes", "k_win", "v_win")]
    w = torch.rand(4, 2, 400, generator=gen(2)).cuda()
    same = w.clone()
    lens = torch.tensor([100, 401, 100, -1], dtype=torch.int32, device="cuda")
    p.slots[2] = 4
    batch = p.cache.batch(p.page_table, lens, torch.zeros(5, dtype=torch.int32, device="cuda"), 0, 0, 400, slots=p.slots)
    p.page_table[0, 0] = -3                 # sources and destinations of tokens 0..15
    kept, lens_out, _ = p.cache.evict(batch, w, 50, 0, 40)
    assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_BATCH | B.SKVQ_STATUS_BAD_PAGE
    assert lens_out.tolist() == [50, 401, 100, -1] and (kept[1:] == -1).all()
    assert torch.equal(w[1:], same[1:])
    pt = p.page_table.cpu().long()
    for x, y in zip(before[:2], (p.cache.k_codes, p.cache.v_codes)):
        for t in range(16, 50):             # the rows that have a page on both sides are right
            for h in range(2):
                old = int(kept[0, h, t])
                if old >= 16:
                    assert torch.equal(y[pt[0, t // 16], h, t % 16], x[pt[0, old // 16], h, old % 16])
        assert torch.equal(x[pt[1:].flatten()], y[pt[1:].flatten()])
    for x, y in zip(before[2:], (p.cache.k_win, p.cache.v_win)):
        assert torch.equal(bits(x[1:]), bits(y[1:]))


@pytest.mark.parametrize("L,keep,levels", [(100003, 50021, 3), (100003, 99999, 1), (262147, 2048, 1 << 20), (40000, 1, 2), (5000, 4999, 2)])
def test_selection_over_long_sequences(L, keep, levels):
    """Kept tokens of long sequences, from few distinct weights to nearly none alike; the order of equal ones."""
    H, P = 3, 256
    n = -(-L // P)
    cache = B.SkvqPagedCache(3, H, 64, 64, 0, P, n, 1)
    g = torch.Generator(device="cuda").manual_seed(L)
    for name in ("k_codes", "v_codes"):
        getattr(cache, name).copy_(torch.randint(0, 256, cache.k_codes.shape, generator=g, device="cuda", dtype=torch.uint8))
    w = torch.floor(torch.rand(1, H, L + 1, generator=g, device="cuda") * levels)
    table = torch.randperm(n, generator=g, device="cuda").int()[None]
    rows = [getattr(cache, name)[table[0].long()].transpose(0, 1).flatten(1, 2)[:, :L].clone() for name in ("k_codes", "v_codes")]
    batch = cache.batch(table, torch.tensor([L], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), 0, 0, L)
    first, recent = (0, 0) if keep < 100 else (5, 40)
    middle = w[:, :, first:L - recent].clone()
    kept, lens_out, _ = cache.evict(batch, w.clone(), keep, first, recent)
    best = torch.sort(middle[0], dim=-1, descending=True, stable=True).indices[:, :keep - first - recent].sort(-1).values + first
    ends = torch.arange(L, device="cuda")
    want = torch.cat((ends[:first].expand(H, -1), best, ends[L - recent:].expand(H, -1)), 1) if recent or first else best
    assert torch.equal(kept[0].long(), want) and int(lens_out[0]) == keep
    for x, name in zip(rows, ("k_codes", "v_codes")):
        now = getattr(cache, name)[table[0].long()].transpose(0, 1).flatten(1, 2)[:, :keep]
        assert torch.equal(now, x.gather(1, want[..., None].expand(-1, -1, x.shape[2])))


@pytest.mark.parametrize("kw", [dict(D=128, G=32, P=16, W=32, R=37), dict(D=64, G=64, H=3, Hq=3, P=32, W=0)])
def test_evict_writes_nothing_beside_its_buffers(kw):
    """Every buffer between guard regions, the workspace of the exact size; bytes behind the new lengths keep what they held."""
    p = GuardedPaged(n_seqs=3, seed=12, max_len=320, **kw)
    p.append([300, 10, 77])
    c, f, guards = p.cache, p.cache.cfg, p.guards
    lens, keep = p.lens(), 64
    w = guarded(torch.rand(3, p.H, 301, generator=gen(4)).cuda(), guards, "weights")
    before, codes = w.clone(), c.k_codes.clone()
    batch = p.batch([0, 0, 0], lens)
    kept, lens_out, first = (guarded(torch.full(s, 9, dtype=torch.int32, device="cuda"), guards, n) for n, s in (("kept", (3, p.H, keep)), ("lens out", (3,)), ("ring from", (3,))))
    size = B.skvq_paged_evict_workspace_size(f, batch)
    ws = guarded(torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda"), guards, "workspace")
    args = B.SkvqPagedEvictArgs(keep, 3, 32, 301, w.data_ptr(), w.data_ptr(), None, 0, None, lens_out.data_ptr(), first.data_ptr(), kept.data_ptr(), ws.data_ptr(), size)
    B.skvq_paged_evict(f, c.struct, batch, args)
    p.check_guards("evict")
    assert lens_out.tolist() == [64, 10, 64] and torch.equal(w[:, :, 64:], before[:, :, 64:]) and torch.equal(w[1], before[1])
    pt = p.page_table.long()
    for b in (0, 2):      # rows behind the new length
        for t in range(64, lens[b]):
            assert torch.equal(c.k_codes[pt[b, t // p.P], :, t % p.P], codes[pt[b, t // p.P], :, t % p.P])
    assert torch.equal(c.k_codes[pt[1]], codes[pt[1]])


def test_some_pages_in_place_others_fresh():
    p = base.Paged(n_seqs=2, seed=15, W=16, R=16, P=16, H=3, Hq=3, spare=20, max_len=320)
    p.append([310, 200])
    w = torch.rand(2, 3, 320, generator=gen(9)).cuda()
    table_out = p.page_table[:, :8].contiguous()
    table_out[0, 1], table_out[0, 4], table_out[1, 0], table_out[1, 7] = 3, 0, 11, 7      # spare pages, that nobody reads
    mine = [[plain.chosen(w[b, h].tolist(), L, 120, 5, 20) for h in range(3)] for b, L in enumerate(p.lens())]
    kept, lens_out, ring_from = p.cache.evict(p.batch([0, 0], p.lens()), w, 120, 5, 20, page_table_out=table_out)
    assert kept.tolist() == mine
    for b in range(2):
        shrink(p.ref, b, mine[b])
    check_rows(p, table_out, [0, 1], lens_out, ring_from)


def test_a_sequence_without_evictions_moves_to_another_slot():
    p = base.Paged(n_seqs=2, seed=14, W=16, R=24, slots=[0, 3])
    p.append([50, 9])
    w = torch.rand(4, 2, 60, generator=gen(8)).cuda()
    slots_out = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    old = w.clone()
    kept, lens_out, ring_from = p.cache.evict(p.batch([0, 0], p.lens()), w, 64, 0, 16, slots_out=slots_out)
    assert lens_out.tolist() == [50, 9] and ring_from.tolist() == [26, 0]
    assert torch.equal(w[1, :, :50], old[0, :, :50]) and torch.equal(w[2, :, :9], old[3, :, :9]) and torch.equal(w[0], old[0])
    check_rows(p, p.page_table, [1, 2], lens_out, ring_from)


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("kw", [dict(D=128, G=64, H=2, Hq=4, P=16, W=32, R=40), dict(D=64, G=32, H=2, Hq=8, P=16, W=16, dtype=BF16)])
def test_a_run_of_all_of_them(kw):
    """Prompts with pictures: rotate by time, height and width, append, attend, weigh, evict; then decode the same way, positions
    running on while the cache stays short."""
    p = Weighed(n_seqs=2, seed=81, capacity=401, **kw)
    D, first, recent, keep = p.D, 2, 40, 70
    table = ref.table64(D, 600).float()
    rope, of_pair = B.RopeTable(table.cuda(), D), [j % 3 for j in range(D // 2)]
    axes = B.RopeAxes(of_pair)
    w, place = torch.full((2, p.H, 401), math.nan), [0, 0]
    wd, position = w.cuda(), [0, 0]
    for step, new in enumerate([[120, 65], [1, 1], [1, 1], [9, 2], [1, 60], [1, 1]]):
        T = sum(new)
        k, v = p.keys(T)
        q = torch.randn(T, p.Hq, D, generator=p.g).to(p.dtype)
        pos = torch.cat([torch.arange(a, a + n) for a, n in zip(position, new)])
        pos = torch.stack((pos, pos // 8, pos % 8)).int()
        position = [a + n for a, n in zip(position, new)]
        qd, kd = q.cuda(), k.cuda()
        rope.apply_axes(axes, pos.cuda(), qd, None, kd, None)
        cs = plain.axis_angles(table, pos, of_pair)
        q, k = ref.rotate32(q, cs, D, False), ref.rotate32(k, cs, D, False)
        assert torch.equal(bits(qd.cpu()), bits(q)) and torch.equal(bits(kd.cpu()), bits(k))
        lens = [a + n for a, n in zip(p.lens(), new)]
        batch = p.batch(new, lens)
        p.cache.append(batch, kd, v.cuda())
        at = 0
        for b, n in enumerate(new):
            p.ref.append(b, k[at:at + n], v[at:at + n])
            at += n
        lse = torch.empty(T, p.Hq, device="cuda")
        out = p.cache.attention(batch, qd, D ** -0.5, lse=lse)
        p.cache.accumulate_weights(batch, qd, lse, wd, D ** -0.5)
        at = 0
        for b, n in enumerate(new):
            want, _, err, _ = p.ref.attention(b, q[at:at + n], D ** -0.5)
            assert ((out[at:at + n].cpu().double() - want).abs() <= err).all(), (step, b)
            want, err = plain.weights(p.ref, b, q[at:at + n], lse[at:at + n].cpu(), w[b], D ** -0.5)
            assert ((wd[b, :, :lens[b]].cpu().double() - want).abs() <= err).all(), (step, b)
            at += n
        w = wd.cpu().clone()
        kept, lens_out, ring_from = p.cache.evict(p.batch([0, 0], lens), wd, keep, first, recent)
        for b, L in enumerate(lens):
            mine = [plain.chosen(w[b, h].tolist(), L, keep, first, recent) for h in range(p.H)]
            assert [[t for t in row if t >= 0] for row in kept[b].cpu().tolist()] == mine
            shrink(p.ref, b, mine)
        w = wd.cpu().clone()
        check_rows(p, p.page_table, [0, 1], lens_out, ring_from)
    assert int(p.cache.status[0]) == 0 and max(p.lens()) == keep


def test_captured_steps_and_other_streams():
    """Weights and eviction captured once, replayed on new queries and from another stream: the eager calls' results; two captured
    graphs do not share anything."""
    H, Hq, D, P, n = 4, 16, 128, 64, 3
    g = torch.Generator(device="cuda").manual_seed(9)
    lens_now = [1500, 700, 64]
    cache = B.SkvqPagedCache(Hq, H, D, 64, 64, P, 3 * 24 * 2, 6)
    for name in ("k_codes", "v_codes"):
        getattr(cache, name).copy_(torch.randint(0, 256, cache.k_codes.shape, generator=g, device="cuda", dtype=torch.uint8))
    for name in ("k_meta", "v_meta", "k_win", "v_win"):
        getattr(cache, name).copy_(torch.rand(getattr(cache, name).shape, generator=g, device="cuda") * 0.2)
    table = torch.randperm(3 * 24, generator=g, device="cuda").int().view(3, 24)
    table_out = table + 3 * 24
    slots, slots_out = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    lens = torch.tensor(lens_now, dtype=torch.int32, device="cuda")
    for rows in (1, 33):
        starts = torch.arange(n + 1, dtype=torch.int32, device="cuda") * rows
        batch = cache.batch(table, lens, starts, n * rows, rows, 1500, slots=slots)
        q, lse = torch.randn(n * rows, Hq, D, generator=g, device="cuda").half(), torch.full((n * rows, Hq), 7.0, device="cuda")
        old = torch.rand(6, H, 1500, generator=g, device="cuda")

        def step():
            w = cache.accumulate_weights(batch, q, lse, old, 0.1, out=torch.zeros_like(old))
            return (w, *cache.evict(batch, w, 600, 4, 100, weights_out=torch.zeros_like(w), page_table_out=table_out, slots_out=slots_out))
        step()
        torch.cuda.synchronize()
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                result = step()
            graphs.append((graph, result))
        side = torch.cuda.Stream()
        for turn in range(3):
            q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
            cache.k_codes[table_out.long()] = 0          # rows behind the new lengths are not written
            want = [x.clone() for x in step()]
            rows_now = cache.k_codes[table_out.long()].clone()
            cache.k_codes[table_out.long()] = 0
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graphs[turn % 2][0].replay()
            side.synchronize()
            for x, y in zip(graphs[turn % 2][1], want):
                assert torch.equal(x, y)
            assert torch.equal(cache.k_codes[table_out.long()], rows_now)
            w = torch.zeros_like(old)
            side.wait_stream(torch.cuda.current_stream())
            got = cache.accumulate_weights(batch, q, lse, old, 0.1, out=w, stream=side)
            side.synchronize()
            assert torch.equal(got, want[0])
    assert int(cache.status[0]) == 0
