"""Out-of-bounds writes of the rotary and paged calls: every buffer they receive sits between patterned guard regions that must
survive, the workspace among them, of exactly the size that skvq_paged_workspace_size gives; and what a call has no business with
keeps its bytes."""
import math

import pytest
import torch

import paged_reference as ref
import test_gpu_rope_paged as base
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build
from test_gpu_guards import Guarded

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
POOL = ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


def guarded(t, guards, name):
    """A copy of t between guard regions."""
    g = Guarded(t.numel() * t.element_size())
    guards[name] = g
    out = g.view(t.dtype, t.shape)
    out.copy_(t)
    return out


class GuardedPaged(base.Paged):
    def __init__(self, **kw):
        super().__init__(**kw)
        self.guards = {}
        c = self.cache
        buffers = {n: guarded(getattr(c, n), self.guards, n) for n in POOL if getattr(c, n).numel()}
        f = c.cfg
        self.cache = B.SkvqPagedCache(f.n_q_heads, f.n_kv_heads, f.head_dim, f.group_size, f.window, f.page_tokens, f.n_pages, f.n_slots, self.dtype,
                                      c.reorder_k, c.reorder_v, c.alpha_k, c.alpha_v, ring_tokens=f.ring_tokens, buffers=buffers)
        c = self.cache
        for n in ("reorder_k", "reorder_v", "alpha_k", "alpha_v", "status"):
            if getattr(c, n) is not None:
                setattr(c, n, guarded(getattr(c, n), self.guards, n))
        c.struct = B.SkvqPagedCacheStruct(*[None if t is None or not t.numel() else t.data_ptr() for t in (
            c.k_codes, c.v_codes, c.k_meta, c.v_meta, c.k_win, c.v_win, c.reorder_k, c.reorder_v, c.alpha_k, c.alpha_v, c.status)])
        if self.rope:
            self.rope = B.RopeTable(guarded(self.rope.table, self.guards, "table"), self.rope.rot_dim, self.rope.interleaved)

    def batch(self, *a, **kw):
        b = super().batch(*a, **kw)
        kept = [None if t is None else guarded(t, self.guards, n) for n, t in zip(("page_table", "lens", "starts", "slots"), b.keep)]
        return self.cache.batch(*kept[:3], b.n_tokens, b.max_new, b.max_len, slots=kept[3])

    def check_guards(self, what):
        torch.cuda.synchronize()
        for name, g in self.guards.items():
            assert g.margins_intact(), f"{what}: bytes next to {name} were overwritten"

    def step(self, new, n_splits=0, causal=True):
        """Append, read and attention of a step, every operand guarded, a workspace of the exact size."""
        T = sum(new)
        k, v = self.keys(T)
        lens = [a + n for a, n in zip(self.lens(), new)]
        b = self.batch(new, lens)
        self.cache.append(b, guarded(k.cuda(), self.guards, "k"), guarded(v.cuda(), self.guards, "v"), rope=self.rope)
        at = 0
        for i, n in enumerate(new):
            self.ref.append(i, k[at:at + n], v[at:at + n])
            at += n
        self.check_guards("append")
        for window in (True, False):
            ko, vo = (guarded(torch.full((T, self.H, self.D), math.nan, dtype=self.dtype, device="cuda"), self.guards, n) for n in ("k out", "v out"))
            self.cache.read(b, ko, vo, window=window)
            self.check_guards("read")
            assert torch.isfinite(ko.float()).all() and torch.isfinite(vo.float()).all()
        q = torch.randn(T, self.Hq, self.D, generator=self.g).to(self.dtype)
        need = B.skvq_paged_workspace_size(self.cache.cfg, b, n_splits)
        self.guards.pop("workspace", None)
        ws = None
        if need:
            self.guards["workspace"] = Guarded(need, fill=0xFF)      # NaN: what a kernel reads before it is written spoils a row
            ws = self.guards["workspace"].body
        out = guarded(torch.full((T, self.Hq, self.D), 9.0, dtype=self.dtype, device="cuda"), self.guards, "out")
        lse = guarded(torch.full((T, self.Hq), 9.0, device="cuda"), self.guards, "lse")
        qd = guarded(q.cuda(), self.guards, "q")
        self.cache.attention(b, qd, 1 / math.sqrt(self.D), out=out, causal=causal, rope=self.rope, lse=lse, n_splits=n_splits, workspace=ws)
        self.check_guards("attention")
        if need:
            with pytest.raises(B.SkvqError) as e:
                self.cache.attention(b, qd, 0.1, out=out, n_splits=n_splits, workspace=ws[:need - 1])
            assert e.value.code == B.SKVQ_ERR_WORKSPACE
        at = 0
        for i, n in enumerate(new):
            want, wl, err, el = self.ref.attention(i, q[at:at + n], 1 / math.sqrt(self.D), causal)
            assert ((out[at:at + n].cpu().double() - want).abs() <= err).all(), i
            assert ((lse[at:at + n].cpu().double() - wl).abs() <= el).all(), i
            at += n
        return need


@pytest.mark.parametrize("kw", base.SHAPES)
def test_paged_calls_write_nothing_outside_their_buffers(kw):
    p = GuardedPaged(n_seqs=3, seed=211, slots=[2, 0, 1], max_len=1500, **kw)
    sizes = [p.step(new, n_splits, causal) for new, n_splits, causal in (
        ([700, 33, 1], 0, True), ([1, 1, 1], 0, True), ([1, 1, 1], 3, True), ([2, 1, 3], 0, False), ([17, 130, 1], 2, True), ([1, 2, 300], 0, True))]
    assert any(sizes)
    p.check_rows()
    assert int(p.cache.status[0]) == 0


def test_rotary_calls_write_nothing_outside_their_buffers():
    for rot, D, dtype, inter, shift in ((128, 128, F16, False, 0), (64, 128, BF16, True, 0), (6, 10, F32, False, 1), (34, 67, F16, True, 1), (256, 512, F32, True, 0)):
        guards = {}
        n, T, H = 77, 13, 3
        f, amp = B.skvq_rope_frequencies(rot, B.SkvqRopeScaling(0, 4096, 10000.0, 1.0, 32.0, 1.0))
        table = guarded(torch.zeros(n, rot // 2, 2, device="cuda"), guards, "table")
        B.skvq_rope_table(f, amp, 0, n, table)
        rope = B.RopeTable(table, rot, inter)
        g = torch.Generator().manual_seed(rot)
        x = torch.randn(T, H, D, generator=g).to(dtype)
        pos = torch.randint(0, n, (T,), generator=g).int()
        pos[4] = n
        status = guarded(torch.zeros(1, dtype=torch.int32, device="cuda"), guards, "status")
        flat = guarded(torch.full((T * H * D + shift,), 3.0, dtype=dtype, device="cuda"), guards, "y")
        y = flat[shift:].view(T, H, D)
        k = guarded(x.cuda(), guards, "k")
        rope.apply(guarded(pos.cuda(), guards, "positions"), guarded(x.cuda(), guards, "x"), y, k, status=status)
        torch.cuda.synchronize()
        for name, gd in guards.items():
            assert gd.margins_intact(), f"bytes next to {name} were overwritten"
        want = ref.rotate32(x, table.cpu()[pos.long().clamp(max=n - 1)], rot, inter)
        kept = torch.arange(T) != 4
        for got in (y, k):
            assert torch.equal(base.bits(got.cpu()[kept]), base.bits(want[kept]))
        assert (y[4] == 3).all() and torch.equal(k[4].cpu(), x[4]) and (flat[:shift] == 3).all()
        assert int(status.item()) == B.SKVQ_STATUS_BAD_POSITION


def test_a_broken_sequence_and_idle_ones_keep_their_bytes():
    """Sequence 0 has three new rows, sequence 1's rows run backwards, 2 and 3 are idle: append writes the first one's three tokens and
    nothing else; append, read and attention each report the second."""
    p = base.Paged(n_seqs=4, seed=221, rot=128, max_len=200)
    p.append([40, 41, 42, 43])
    T = 12
    k, v = p.keys(T)
    q = torch.randn(T, 4, 128, generator=p.g).half()
    b = p.cache.batch(p.page_table, torch.tensor([43, 41, 42, 43], dtype=torch.int32, device="cuda"), torch.tensor([0, 3, 0, 0, 0], dtype=torch.int32, device="cuda"), T, 4, 200)

    def status():
        got = int(p.cache.status[0])
        p.cache.status.zero_()
        return got

    p.cache.append(b, k.cuda(), v.cuda(), rope=p.rope)
    assert status() == B.SKVQ_STATUS_BAD_BATCH
    p.ref.append(0, k[:3], v[:3])
    p.check_rows()                               # sequence 0's new rows, and every other byte of pages and ring as it was
    ko, vo = (torch.full((T, 2, 128), 9.0, dtype=F16, device="cuda") for _ in range(2))
    p.cache.read(b, ko, vo)
    assert status() == B.SKVQ_STATUS_BAD_BATCH
    assert (ko[:3] != 9).any(-1).all() and (ko[3:] == 9).all() and (vo[3:] == 9).all()
    out = torch.full((T, 4, 128), 9.0, dtype=F16, device="cuda")
    p.cache.attention(b, q.cuda(), 0.1, out=out, rope=p.rope)
    assert status() == B.SKVQ_STATUS_BAD_BATCH
    want, _, err, _ = p.ref.attention(0, q[:3], 0.1)
    assert ((out[:3].cpu().double() - want).abs() <= err).all() and (out[3:] == 9).all()
