"""Sizing and refusals of the paged and rotary calls at the ends of their ranges: host only, nothing is launched."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import test_rope_paged_host as base
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build

FAKE = 0x1000
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.lib()


def batch(**kw):
    fields = dict(page_table=FAKE, lens=FAKE, starts=FAKE, slots=None, n_seqs=3, max_pages=5, n_tokens=7, max_new=4, max_len=320)
    fields.update(kw)
    return B.SkvqPagedBatch(**fields)


def three_calls(lib, b, cfg=None):
    """Codes of append, read and attention for a batch; everything else is in order."""
    c = ctypes.byref(base.pcfg(**(cfg or {})))
    p = ctypes.byref(B.SkvqPagedCacheStruct(k_codes=FAKE, v_codes=FAKE, k_meta=FAKE, v_meta=FAKE, k_win=FAKE, v_win=FAKE))
    a = ctypes.byref(B.SkvqPagedAttnArgs(0.1, 1, 0, FAKE, 1 << 40))
    b = ctypes.byref(b)
    return [lib.skvq_paged_append(c, p, b, None, FAKE, FAKE, 1024, 1024, None), lib.skvq_paged_read(c, p, b, 1, FAKE, FAKE, 1024, 1024, None),
            lib.skvq_paged_attention(c, p, b, None, FAKE, 1024, FAKE, 1024, None, a, None)]


def test_first_ring_tokens_are_checked(lib):
    before = B.skvq_launch_count()
    assert three_calls(lib, batch(ring_from=FAKE + 2)) == [B.SKVQ_ERR_MISALIGNED] * 3
    assert B.skvq_launch_count() == before


def run(code):
    return subprocess.run([sys.executable, "-c", "from paper_2405_06219_b200 import binding as B\n" + code], cwd=ROOT, capture_output=True, text=True)


@pytest.mark.parametrize("kw", [dict(max_new=0, n_tokens=0), dict(max_new=0, n_tokens=7), dict(max_new=4, n_tokens=0)])
def test_a_step_without_new_tokens_needs_no_workspace(lib, kw):
    """In a process of its own: the sizing once divided by the number of items."""
    code = """
cfg = B.SkvqPagedConfig(32, 8, 128, 64, 128, 128, 64, 4000, 4, 0)
for max_len in (0, 128, 4096, 200000):
    for n_splits in (0, 1, 5):
        assert B.skvq_paged_workspace_size(cfg, B.SkvqPagedBatch(n_seqs=1, max_pages=4000, max_len=max_len, **%r), n_splits) == 0
""" % kw
    r = run(code)
    assert r.returncode == 0, (r.returncode, r.stderr)


def test_sizing_refuses_what_the_calls_refuse(lib):
    cfg = base.pcfg()
    long = dict(max_pages=5000, max_len=300000)
    assert B.skvq_paged_workspace_size(cfg, batch(**long)) > 0
    for kw in (dict(max_new=-1), dict(n_tokens=-1), dict(max_len=-1), dict(n_seqs=0), dict(n_seqs=2049)):
        assert B.skvq_paged_workspace_size(cfg, batch(**{**long, **kw})) == 0, kw
    assert B.skvq_paged_workspace_size(cfg, batch(**long), -1) == 0


def test_lengths_whose_token_numbers_would_pass_32_bits_are_refused(lib):
    """Kernels look some 64 blocks of 16 tokens past the length: near 2^31 those numbers would wrap."""
    before = B.skvq_launch_count()
    most = 1 << 30
    for max_len in (most + 1, 2 ** 31 - 1):
        b = batch(max_len=max_len, max_pages=2 ** 31 // 64)
        assert three_calls(lib, b) == [B.SKVQ_ERR_UNSUPPORTED] * 3
        assert B.skvq_paged_workspace_size(base.pcfg(), b) == 0
    assert B.skvq_paged_workspace_size(base.pcfg(), batch(max_len=most, max_pages=most // 64)) > 0
    assert B.skvq_launch_count() == before


def test_a_table_that_begins_beyond_64_bits_is_refused(lib):
    f = (ctypes.c_double * 4)(*[0.5] * 4)
    before = B.skvq_launch_count()
    for first, n in ((2 ** 63 - 1, 1), (2 ** 63 - 10, 100), (2 ** 31 - 1, 1), (2 ** 31 - 5, 5)):
        assert lib.skvq_rope_table(f, 4, 1.0, first, n, FAKE, None) == B.SKVQ_ERR_UNSUPPORTED, (first, n)
    assert B.skvq_launch_count() == before


def test_outputs_whose_rows_overlap_are_refused(lib):
    """Heads or tokens that share a row of y: broadcast outputs, and tensors rotated in place through other strides than x's."""
    before = B.skvq_launch_count()

    def call(x, y, xs, ys, heads=8, T=4, D=128):
        rope = B.SkvqRope(FAKE, 64, 0, 8)
        a = B.SkvqRopeTensor(x, y, *xs, *ys, heads)
        ok = B.SkvqRopeTensor(FAKE, FAKE + (1 << 20), 1024, 128, 1024, 128, 8)
        return [lib.skvq_rope_apply(ctypes.byref(rope), B.SKVQ_F16, D, ctypes.byref(p), ctypes.byref(q), FAKE, T, 0, None, None) for p, q in ((a, ok), (ok, a))]

    bad = [B.SKVQ_ERR_INVALID_ARG] * 2
    far = FAKE + (1 << 24)
    assert call(FAKE, far, (1024, 128), (1024, 0)) == bad             # every head into one row
    assert call(FAKE, far, (1024, 128), (0, 128)) == bad              # every token into one row
    assert call(FAKE, far, (1024, 128), (1024, 64)) == bad            # heads that reach into each other
    assert call(FAKE, far, (1024, 128), (1024, -64)) == bad
    assert call(FAKE, far, (1024, 128), (127, 128), heads=1) == bad
    assert call(FAKE, far, (1024, 128), (128, 128)) == bad            # a token's second head is the next token's first
    assert call(FAKE, far, (1024, 128), (-384, 128)) == bad
    assert call(FAKE, far, (1024, 128), (2 ** 62, 2 ** 62 + 64)) == bad
    assert call(FAKE, FAKE, (1024, 0), (1024, 0)) == bad              # a broadcast input in place
    assert call(FAKE, FAKE, (1024, 128), (1024, 256)) == bad          # in place, other strides
    assert call(FAKE, FAKE, (1024, 128), (2048, 128)) == bad
    assert B.skvq_launch_count() == before


# ------------------------------------------------------------------------------------------------ tensors of another GPU, in the binding
class OnGpu:
    """What the binding asks of a tensor, on a GPU that need not exist."""

    def __init__(self, index, shape, dtype):
        self.index, self.shape, self.dtype = index, shape, dtype

    def get_device(self):
        return self.index

    def stride(self):
        out = [1]
        for n in self.shape[:0:-1]:
            out.insert(0, out[0] * n)
        return tuple(out)

    def data_ptr(self):
        return FAKE

    def is_contiguous(self):
        return True

    def numel(self):
        n = 1
        for m in self.shape:
            n *= m
        return n


def fake_cache(index):
    c = B.SkvqPagedCache.__new__(B.SkvqPagedCache)
    c.cfg, c.struct, c.dtype, c.index, c.device = base.pcfg(), B.SkvqPagedCacheStruct(), torch.float16, index, torch.device("cuda", index)
    return c


def fake_rope(index):
    r = B.RopeTable.__new__(B.RopeTable)
    r.struct, r.rot_dim, r.interleaved, r.index = B.SkvqRope(FAKE, 64, 0, 8), 64, False, index
    return r


def test_a_rotation_of_another_gpu_is_refused():
    c = fake_cache(1)
    k, q = OnGpu(1, (7, 2, 128), torch.float16), OnGpu(1, (7, 8, 128), torch.float16)
    for call in (lambda rope: c.append(batch(), k, k, rope=rope),
                 lambda rope: c.attention(batch(), q, 0.1, out=q, rope=rope)):
        with pytest.raises(AssertionError, match="rotation"):
            call(fake_rope(0))


def test_a_batch_of_another_gpu_is_refused():
    c, b = fake_cache(1), batch()
    b.index = 0
    k, q = OnGpu(1, (7, 2, 128), torch.float16), OnGpu(1, (7, 8, 128), torch.float16)
    for call in (lambda: c.append(b, k, k), lambda: c.read(b, k, k), lambda: c.attention(b, q, 0.1, out=q)):
        with pytest.raises(AssertionError, match="batch"):
            call()


@pytest.mark.parametrize("status", [OnGpu(1, (1,), torch.int32), OnGpu(0, (1,), torch.int64), OnGpu(0, (0,), torch.int32)])
def test_a_status_word_that_is_none_is_refused(status):
    pos, x = OnGpu(0, (7,), torch.int32), OnGpu(0, (7, 2, 128), torch.float16)
    with pytest.raises(AssertionError, match="status"):
        fake_rope(0).apply(pos, x, status=status)
