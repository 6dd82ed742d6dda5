"""The paged cache where it meets an engine's own bookkeeping: kept prefixes, sequences that change their slot, page-table entries
that are no pages, queries that are not finite.  Against the plain 64-bit forms of paged_reference, with their counted bounds."""
import math
import threading

import pytest
import torch

import paged_reference as ref
import test_gpu_rope_paged as base
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


# ------------------------------------------------------------------------------------------------ a window that reaches back behind the ring
class FromPages(ref.Reference):
    """The plain cache with a first ring token per sequence: tokens before it are read from their pages, inside the window too."""

    def __init__(self, plain, n):
        self.__dict__.update(plain.__dict__)
        self.ring_from = [0] * n

    def ring_rows(self, b):
        L = len(self.rows[b])
        return min(self.W, L - min(max(self.ring_from[b], 0), L))

    def values(self, b, which, window=True):
        whole, self.W = self.W, self.ring_rows(b)
        try:
            return super().values(b, which, window)
        finally:
            self.W = whole

    def score_error(self, b):
        whole, self.W = self.W, self.ring_rows(b)
        try:
            return super().score_error(b)
        finally:
            self.W = whole


class Engine(base.Paged):
    """A cache whose sequences say where their ring begins; ring rows that nobody wrote are NaN."""

    def __init__(self, n_seqs, **kw):
        super().__init__(n_seqs=n_seqs, **kw)
        self.ref = FromPages(self.ref, n_seqs)

    def batch(self, new, lens, pad=0, max_new=None, max_len=None):
        b = super().batch(new, lens, pad, max_new, max_len)
        first = torch.tensor(self.ref.ring_from, dtype=torch.int32, device="cuda")
        return self.cache.batch(*b.keep[:3], b.n_tokens, b.max_new, b.max_len, slots=b.keep[3], ring_from=first)

    def check_read(self, new):
        """The last rows of every sequence as attention sees them."""
        T = sum(new)
        k, v = self.cache.read(self.batch(new, self.lens()))
        at = 0
        for i, n in enumerate(new):
            L = len(self.ref.rows[i])
            for got, which, idx in ((k, "k", self.ref.rk), (v, "v", self.ref.rv)):
                val = self.ref.values(i, which)[L - n:].float().to(self.dtype)
                want = torch.empty(n, self.H, self.D, dtype=self.dtype)
                for h in range(self.H):
                    want[:, h, idx[h]] = val[:, h]
                assert torch.equal(base.bits(got[at:at + n].cpu()), base.bits(want)), (i, which)
            at += n
        assert at == T


RINGS = [dict(W=32, P=32, D=128, G=64, rot=64), dict(W=20, R=33, P=16, D=64, G=32, H=3, Hq=9, dtype=BF16), dict(W=150, P=16, D=128, G=32, H=1, Hq=4, rot=128, inter=True)]


@pytest.mark.parametrize("kw", RINGS)
def test_a_kept_prefix_under_a_window(kw):
    """A second sequence begins on the first one's pages: the prefix tokens of its window are read from there, until the window has
    passed them."""
    p = Engine(2, seed=71, **kw)
    p.append([96, 0])
    shared = 96 // p.P
    p.page_table[1, :shared] = p.page_table[0, :shared]
    p.ref.rows[1] = list(p.ref.rows[0])
    p.ref.ring_from[1] = 96
    p.check_attention([1, 1])                    # nothing appended yet: the whole window lies in shared pages
    p.check_attention([90, 60])
    for new in ([1, 1], [3, 2], [10, 14], [1, 1], [40, 60], [1, 1], [90, 100]):
        p.append(new)
        p.check_attention(new)
        p.check_attention([1, 1], n_splits=2)
        p.check_attention([30, 50], causal=False)
        p.check_read([min(60, n) for n in p.lens()])
    assert int(p.cache.status[0]) == 0


@pytest.mark.parametrize("kw", RINGS)
@pytest.mark.parametrize("length", [1, 15, 37, 130])
def test_a_sequence_that_comes_back_in_another_slot(kw, length):
    p = Engine(2, seed=72, slots=[0, 1, 2, 3], **kw)
    p.slots = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    p.append([length, 50])
    p.slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")      # slot 3 was never written
    p.ref.ring_from[0] = length
    p.check_attention([1, 1])
    for new in ([1, 1], [17, 1], [64, 30]):
        p.append(new)
        p.check_attention(new)
        p.check_attention([1, 4])
        p.check_read([min(5, n) for n in p.lens()])
    assert int(p.cache.status[0]) == 0


def test_first_ring_tokens_outside_the_sequence():
    p = Engine(3, W=32, seed=73)
    p.append([100, 40, 0])
    p.cache.k_win[1].fill_(math.nan)             # all of this one comes from its pages
    p.cache.v_win[1].fill_(math.nan)
    p.ref.ring_from = [-7, 2 ** 31 - 1, 5]
    p.check_attention([1, 1, 1])
    p.check_attention([50, 40, 0])
    p.check_read([60, 40, 0])
    assert int(p.cache.status[0]) == 0


def test_taking_back_more_than_the_ring_holds():
    """The ring is as long as the window: tokens that were refused took the rows of older ones, which then come from their pages."""
    p = Engine(1, W=32, seed=74, max_len=200)
    p.append([100])
    p.append([8])
    p.ref.truncate(0, 102)
    p.ref.ring_from = [108 - 32]
    p.check_attention([1])
    p.check_attention([40])
    p.check_read([40])


# ------------------------------------------------------------------------------------------------ a window token without a page
@pytest.mark.parametrize("kw", [dict(D=128, G=64), dict(D=64, G=32, H=1, Hq=4, dtype=BF16)])
@pytest.mark.parametrize("entry", [-1, 2 ** 31 - 1])
@pytest.mark.parametrize("appended", [True, False])
def test_a_bad_page_under_the_window(kw, entry, appended):
    """Tokens 64..79 lose their page, after they were appended or before (then their ring rows were never written): attention leaves
    them out, read leaves their rows alone, both report them.  The window begins inside a page, its tiles straddle the bad one."""
    p = base.Paged(n_seqs=1, W=41, P=16, seed=111, max_len=128, **kw)
    good = p.page_table.clone()
    if appended:
        p.append([100])
    p.page_table[0, 4] = entry
    if not appended:
        p.append([100])
        assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_PAGE
        p.cache.status.zero_()
    without = ref.Reference(1, p.Hq, p.H, p.D, kw["G"], 41 - 16, p.dtype, p.ref.rk, p.ref.rv, p.ref.ak, p.ref.av)
    without.rows[0] = p.ref.rows[0][:64] + p.ref.rows[0][80:]
    for new in (1, 3, 100):
        for causal in (False, True):
            p.cache.status.zero_()
            q = torch.randn(new, p.Hq, p.D, generator=p.g).to(p.dtype)
            lse = torch.empty(new, p.Hq, device="cuda")
            out = p.cache.attention(p.batch([new], [100]), q.cuda(), 0.1, causal=causal, lse=lse)
            assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_PAGE
            for i in {0, min(70, new - 1), new - 1}:
                limit = 100 - new + i + 1 if causal else 100
                kept = limit - max(0, min(limit, 80) - 64)      # of the tokens that are left
                few = ref.Reference(1, p.Hq, p.H, p.D, kw["G"], max(0, kept - (84 - 25)), p.dtype, p.ref.rk, p.ref.rv, p.ref.ak, p.ref.av)
                few.rows[0] = without.rows[0][:kept]
                want, wl, err, el = few.attention(0, q[i:i + 1], 0.1, causal=False)
                assert ((out.cpu().double()[i:i + 1] - want).abs() <= err).all()
                assert ((lse.cpu().double()[i:i + 1] - wl).abs() <= el).all()
    p.cache.status.zero_()
    got, _ = p.cache.read(p.batch([100], [100]), torch.full((100, p.H, p.D), 9.0, dtype=p.dtype, device="cuda"))
    assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_PAGE
    assert (got[64:80] == 9).all() and torch.isfinite(got.float()).all() and not (got[:64] == 9).all(-1).any() and not (got[80:] == 9).all(-1).any()
    p.cache.status.zero_()
    p.page_table.copy_(good)
    if appended:
        p.check_attention([1])
        p.check_attention([100])
        assert int(p.cache.status[0]) == 0


# ------------------------------------------------------------------------------------------------ queries that are not finite
@pytest.mark.parametrize("length,window,new", [(40, 64, 1), (40, 64, 3), (40, 64, 40), (90, 0, 2), (90, 0, 60), (200, 32, 1), (200, 32, 100)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [0.1, -0.1, 0.0])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_an_infinite_query_gives_its_row_nan(length, window, new, dtype, scale, value):
    """Keys of one sign: the scores of an infinite query are all of one sign too, -infinity among them, which means masked elsewhere."""
    p = base.Paged(n_seqs=1, W=window, P=64, seed=191, dtype=dtype)
    k, v = p.keys(length)
    k = k.abs() + 0.25
    p.cache.append(p.batch([length], [length]), k.cuda(), v.cuda())
    p.ref.append(0, k, v)
    q = torch.randn(new, 4, 128, generator=p.g).to(dtype)
    lse = [torch.empty(new, 4, device="cuda") for _ in range(2)]
    good = p.cache.attention(p.batch([new], [length]), q.cuda(), scale, lse=lse[0])
    assert torch.isfinite(good.float()).all()
    q[new - 1, 2, 7] = value
    out = p.cache.attention(p.batch([new], [length]), q.cuda(), scale, lse=lse[1])
    spoilt = torch.zeros(new, 4, dtype=torch.bool, device="cuda")
    spoilt[new - 1, 2] = True
    assert torch.isnan(out[spoilt]).all() and torch.isnan(lse[1][spoilt]).all()
    assert torch.equal(out[~spoilt], good[~spoilt]) and torch.equal(lse[1][~spoilt], lse[0][~spoilt])


def test_an_infinite_query_that_sees_nothing_gives_zeros():
    p = base.Paged(n_seqs=1, seed=192)
    p.append([2])
    for new in (5, 40):
        q = torch.randn(new, 4, 128, generator=p.g).half()
        q[0, 1, 3] = math.inf
        lse = torch.empty(new, 4, device="cuda")
        out = p.cache.attention(p.batch([new], [2]), q.cuda(), 0.1, lse=lse)
        assert (out[0, 1] == 0).all() and float(lse[0, 1]) == -math.inf


def test_a_step_without_new_tokens():
    """A batch over long contexts in which nobody has a new token: nothing to do, in every call."""
    p = base.Paged(n_seqs=2, W=16, P=64, seed=201, max_len=4096)
    p.append([40, 3])
    before = [getattr(p.cache, n).clone() for n in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")]
    none = torch.zeros(0, 2, 128, dtype=F16, device="cuda")
    for max_len in (100, 4096):
        b = p.batch([0, 0], p.lens(), max_len=max_len)
        for n_splits in (0, 4):
            assert p.cache.attention(b, torch.zeros(0, 4, 128, dtype=F16, device="cuda"), 0.1, n_splits=n_splits).shape == (0, 4, 128)
        p.cache.append(b, none, none)
        assert p.cache.read(b)[0].shape == (0, 2, 128)
    torch.cuda.synchronize()
    for x, n in zip(before, ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win")):
        assert torch.equal(x.view(torch.uint8), getattr(p.cache, n).view(torch.uint8)), n
    assert int(p.cache.status[0]) == 0


# ------------------------------------------------------------------------------------------------ rotation of broadcast and strided rows
@pytest.mark.parametrize("inter", [False, True])
def test_rotation_of_a_broadcast_input_and_of_odd_layouts(inter):
    """One head or one token broadcast to many; outputs head by head, backwards, and with rows that interleave without touching."""
    T, H, D, rot = 3, 3, 8, 8
    g = torch.Generator().manual_seed(7)
    cs = ref.table64(rot, 50).float()
    rope = B.RopeTable(cs.cuda(), rot, inter)
    pos = torch.tensor([4, 49, 0], dtype=torch.int32)
    for x in (torch.randn(T, 1, D, generator=g).expand(T, H, D), torch.randn(1, H, D, generator=g).expand(T, H, D), torch.randn(T, H, D, generator=g)):
        want = ref.rotate32(x.contiguous(), cs[pos.long()], rot, inter)
        src = x[:, :1].cuda().expand(T, H, D) if x.stride(1) == 0 else x[:1].cuda().expand(T, H, D) if x.stride(0) == 0 else x.cuda()
        assert src.stride() == x.stride()
        for strides in ((H * D, D, 1), (D, T * D, 1), (16, 24, 1), (40, 16, 1)):
            pool = torch.full((200,), 5.0, device="cuda")
            out = pool.as_strided((T, H, D), strides, 3)
            rope.apply(pos.cuda(), src, out)
            assert torch.equal(base.bits(out.cpu()), base.bits(want)), strides
            written = torch.zeros(200, dtype=torch.bool)
            written.as_strided((T, H, D), strides, 3).fill_(True)
            assert (pool.cpu()[~written] == 5).all(), strides
    with pytest.raises(B.SkvqError) as e:
        rope.apply(pos.cuda(), torch.zeros(T, 1, D, device="cuda").expand(T, H, D))
    assert e.value.code == B.SKVQ_ERR_INVALID_ARG


@pytest.mark.parametrize("new", [1, 3, 60])
def test_the_largest_magnitudes(new):
    """Groups that span +-65440: every value of theirs, and of the operands, still is a finite fp16."""
    p = base.Paged(n_seqs=1, W=16, P=64, seed=231, reorder=False, outliers=False)
    k, v = p.keys(120)
    for x in (k, v):
        x[:, :, 3::32], x[:, :, 5::32] = 65440.0, -65440.0
    p.cache.append(p.batch([120], [120]), k.cuda(), v.cuda())
    p.ref.append(0, k, v)
    p.check_rows()
    ko, vo = p.cache.read(p.batch([120], [120]), window=False)
    assert torch.isfinite(ko.float()).all() and torch.isfinite(vo.float()).all()
    p.check_attention([new], sm_scale=1e-7)


# ------------------------------------------------------------------------------------------------ two calls at once, captured prompts
def test_two_host_threads_and_two_graphs_of_a_prompt_step():
    """Calls from two threads on a stream each, and a step of prompts and single tokens captured twice and replayed side by side with
    lengths that change on the device: every result as it is alone."""
    p = base.Paged(n_seqs=4, Hq=8, H=2, seed=241, W=32, P=32, rot=64)
    p.append([180, 40, 300, 7])
    new = [150, 1, 20, 1]
    q = torch.randn(sum(new), 8, 128, generator=p.g).half().cuda()
    b, one = p.batch(new, p.lens()), p.batch([1, 1, 1, 1], p.lens())
    q1 = q[:4].contiguous()
    alone = [p.cache.attention(b, q, 0.1, rope=p.rope), p.cache.attention(one, q1, 0.1, rope=p.rope)]
    torch.cuda.synchronize()
    got = [[], []]

    def calls(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got[i].append(p.cache.attention(b, q, 0.1, rope=p.rope) if i == 0 else p.cache.attention(one, q1, 0.1, rope=p.rope))
        stream.synchronize()

    threads = [threading.Thread(target=calls, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert len(got[0]) == len(got[1]) == 20
    assert all(torch.equal(x, alone[i]) for i in range(2) for x in got[i])
    lens = torch.tensor(p.lens(), dtype=torch.int32, device="cuda")
    live = p.cache.batch(p.page_table, lens, b.keep[2], sum(new), 150, p.max_pages * p.P)
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(p.cache.attention(live, q, 0.1, rope=p.rope))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for less in (0, 3, 6):
        lens.copy_(torch.tensor([n - less for n in p.lens()], dtype=torch.int32))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    g.replay()
        torch.cuda.synchronize()
        want = p.cache.attention(live, q, 0.1, rope=p.rope)
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    assert int(p.cache.status[0]) == 0


@pytest.mark.parametrize("rows", [1, 17])
def test_a_context_of_sixteen_million_tokens(rows):
    """One page over and over: the answer is that of the page, the log-sum-exp larger by the logarithm of the number of pages."""
    P, D, L = 256, 64, 1 << 24
    p = base.Paged(n_seqs=1, Hq=1, H=1, D=D, G=64, W=0, P=P, max_len=P, seed=251, reorder=False, outliers=False)
    p.append([P])
    q = torch.randn(rows, 1, D, generator=p.g).half()
    table = p.page_table[:, :1].expand(1, L // P).contiguous()
    b = p.cache.batch(table, torch.tensor([L], dtype=torch.int32, device="cuda"), torch.tensor([0, rows], dtype=torch.int32, device="cuda"), rows, rows, L)
    lse = torch.empty(rows, 1, device="cuda")
    out = p.cache.attention(b, q.cuda(), 0.125, causal=False, lse=lse)
    want, wl, err, el = p.ref.attention(0, q, 0.125, causal=False)
    # The longest chain of one accumulator's truncated sums is that of a CTA's warp in the kernel for few rows (2^24 tokens over 148 x 3 CTAs
    # of 4 warps, 16 tokens a product: 591), a CTA's tiles in the other (2^24 over 148 CTAs, 16 tokens a product: 7085).
    chain = 7100 * 2.0 ** -23
    top = float(p.ref.values(0, "v").abs().max())
    assert ((out.cpu().double() - want).abs() <= err + chain * top).all()
    assert ((lse.cpu().double() - wl - math.log(L // P)).abs() <= el + chain + 30 * 2.0 ** -23).all()
    assert int(p.cache.status[0]) == 0
