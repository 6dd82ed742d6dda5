"""Refusals and sizes of the rotation with several axes, of accumulated attention weights and of eviction: host only, nothing is
launched.  Pointers are made up and never dereferenced."""
import ctypes

import pytest
import torch

from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build

FAKE = 0x1000


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.lib()


@pytest.fixture(autouse=True)
def _nothing_launched(lib):
    before = B.skvq_launch_count()
    yield
    assert B.skvq_launch_count() == before


def test_axes_refusals(lib):
    def call(rope=(FAKE, 64, 0, 8), of_pair=(0, 1, 2), n_axes=3, dtype=B.SKVQ_F16, D=128, a=(FAKE, FAKE, 1024, 128, 1024, 128, 8), pos=FAKE, T=4, inv=0,
             status=None, axes=True):
        of = (ctypes.c_uint8 * 128)(*[of_pair[j % len(of_pair)] for j in range(128)])
        ta = None if a is None else ctypes.byref(B.SkvqRopeTensor(*a))
        x = ctypes.byref(B.SkvqRopeAxes(n_axes, of)) if axes else None
        return lib.skvq_rope_apply_axes(ctypes.byref(B.SkvqRope(*rope)), x, dtype, D, ta, None, pos, T, 1, T, inv, status, None)

    assert call(axes=False) == B.SKVQ_ERR_INVALID_ARG
    assert call(n_axes=0) == B.SKVQ_ERR_INVALID_ARG
    assert call(n_axes=5) == B.SKVQ_ERR_UNSUPPORTED
    assert call(n_axes=2) == B.SKVQ_ERR_INVALID_ARG                       # a pair on axis 2
    assert call(of_pair=(0, 255)) == B.SKVQ_ERR_INVALID_ARG
    assert call(rope=(FAKE, 258, 0, 8), D=512, a=(FAKE, FAKE, 4096, 512, 4096, 512, 8)) == B.SKVQ_ERR_UNSUPPORTED      # more pairs than axis[] has
    # what skvq_rope_apply refuses
    assert call(a=None) == B.SKVQ_ERR_INVALID_ARG
    assert call(T=-1) == B.SKVQ_ERR_INVALID_ARG
    assert call(inv=2) == B.SKVQ_ERR_INVALID_ARG
    assert call(dtype=3) == B.SKVQ_ERR_UNSUPPORTED
    assert call(rope=(FAKE, 63, 0, 8)) == B.SKVQ_ERR_INVALID_ARG
    assert call(rope=(None, 64, 0, 8)) == B.SKVQ_ERR_INVALID_ARG
    assert call(pos=None) == B.SKVQ_ERR_INVALID_ARG
    assert call(pos=FAKE + 2) == B.SKVQ_ERR_MISALIGNED
    assert call(status=FAKE + 2) == B.SKVQ_ERR_MISALIGNED
    assert call(a=(FAKE, FAKE, 1024, 128, 1024, 64, 8)) == B.SKVQ_ERR_INVALID_ARG       # rows of y that share elements
    assert call(a=(FAKE, FAKE, 2048, 128, 1024, 128, 8)) == B.SKVQ_ERR_INVALID_ARG      # in place through other strides
    assert call(T=0) == B.SKVQ_OK
    assert call(a=(FAKE, FAKE, 1024, 128, 1024, 128, 0)) == B.SKVQ_OK                   # no heads
    assert call(T=0, of_pair=(0, 9)) == B.SKVQ_ERR_INVALID_ARG                          # refused before there is nothing to do


def test_axes_of_pairs():
    x = B.RopeAxes.runs([3, 1, 4])
    assert (x.pairs, x.n_axes, list(x.struct.axis[:8])) == (8, 3, [0, 0, 0, 1, 2, 2, 2, 2])
    for bad in ([], [4], [-1], [0] * 129):
        with pytest.raises(AssertionError):
            B.RopeAxes(bad)


def structs(cfg=None, pool=None, batch=None):
    c = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, group_size=64, window=128, ring_tokens=160, page_tokens=64, n_pages=10, n_slots=4, dtype=B.SKVQ_F16)
    c.update(cfg or {})
    p = dict(k_codes=FAKE, v_codes=FAKE, k_meta=FAKE, v_meta=FAKE, k_win=FAKE, v_win=FAKE)
    p.update(pool or {})
    b = dict(page_table=FAKE, lens=FAKE, starts=FAKE, slots=None, n_seqs=3, max_pages=5, n_tokens=7, max_new=4, max_len=320)
    b.update(batch or {})
    return B.SkvqPagedConfig(**c), B.SkvqPagedCacheStruct(**p), B.SkvqPagedBatch(**b)


def weights(lib, cfg=None, pool=None, batch=None, rope=None, q=FAKE, stride=1024, lse=FAKE, args=None):
    a = dict(sm_scale=0.1, causal=1, last=0, capacity=320, weights=FAKE, weights_out=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
    a.update(args or {})
    s = [ctypes.byref(x) for x in structs(cfg, pool, batch)]
    r = None if rope is None else ctypes.byref(B.SkvqRope(*rope))
    return lib.skvq_paged_weights(*s, r, q, stride, lse, ctypes.byref(B.SkvqPagedWeightsArgs(**a)), None)


def evict(lib, cfg=None, pool=None, batch=None, args=None):
    a = dict(keep=200, first=4, recent=128, capacity=320, weights=FAKE, weights_out=FAKE, page_table_out=None, max_pages_out=0, slots_out=None,
             lens_out=FAKE, ring_from_out=None, kept=FAKE, workspace=FAKE, workspace_bytes=1 << 20)
    a.update(args or {})
    s = [ctypes.byref(x) for x in structs(cfg, pool, batch)]
    return lib.skvq_paged_evict(*s, ctypes.byref(B.SkvqPagedEvictArgs(**a)), None)


@pytest.mark.parametrize("call", [weights, evict])
def test_common_refusals(lib, call):
    assert call(lib, cfg=dict(head_dim=80)) == B.SKVQ_ERR_UNSUPPORTED
    for name in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win"):
        assert call(lib, pool={name: None}) == B.SKVQ_ERR_INVALID_ARG, name
        assert call(lib, pool={name: FAKE + 8}) == B.SKVQ_ERR_MISALIGNED, name
    for name in ("page_table", "lens"):
        assert call(lib, batch={name: None}) == B.SKVQ_ERR_INVALID_ARG, name
        assert call(lib, batch={name: FAKE + 2}) == B.SKVQ_ERR_MISALIGNED, name
    assert call(lib, batch=dict(n_seqs=0)) == B.SKVQ_ERR_INVALID_ARG
    assert call(lib, batch=dict(n_seqs=2049, slots=FAKE)) == B.SKVQ_ERR_UNSUPPORTED
    assert call(lib, batch=dict(max_len=321)) == B.SKVQ_ERR_CAPACITY                    # five pages of 64
    # without slot numbers a slot per sequence, whatever the window
    assert call(lib, batch=dict(n_seqs=5)) == B.SKVQ_ERR_CAPACITY
    assert call(lib, cfg=dict(window=0, ring_tokens=0), batch=dict(n_seqs=5)) == B.SKVQ_ERR_CAPACITY
    assert call(lib, args=dict(capacity=319)) == B.SKVQ_ERR_CAPACITY
    assert call(lib, args=dict(capacity=0)) == B.SKVQ_ERR_INVALID_ARG
    assert call(lib, args=dict(weights_out=None)) == B.SKVQ_ERR_INVALID_ARG
    for name in ("weights", "weights_out"):
        assert call(lib, args={name: FAKE + 2}) == B.SKVQ_ERR_MISALIGNED, name
    assert call(lib, args=dict(workspace=FAKE + 8)) == B.SKVQ_ERR_MISALIGNED
    rows = dict(n_tokens=70, max_new=40)      # (few rows need no workspace)
    assert call(lib, batch=rows, args=dict(workspace=None)) == B.SKVQ_ERR_WORKSPACE
    assert call(lib, batch=rows, args=dict(workspace_bytes=8)) == B.SKVQ_ERR_WORKSPACE


def test_weights_refusals(lib):
    assert weights(lib, batch=dict(starts=None)) == B.SKVQ_ERR_INVALID_ARG
    assert weights(lib, q=None) == B.SKVQ_ERR_INVALID_ARG and weights(lib, lse=None) == B.SKVQ_ERR_INVALID_ARG
    assert weights(lib, q=FAKE + 2) == B.SKVQ_ERR_MISALIGNED and weights(lib, lse=FAKE + 2) == B.SKVQ_ERR_MISALIGNED
    assert weights(lib, stride=1028) == B.SKVQ_ERR_MISALIGNED and weights(lib, stride=1016) == B.SKVQ_ERR_INVALID_ARG
    assert weights(lib, args=dict(causal=2)) == B.SKVQ_ERR_INVALID_ARG and weights(lib, args=dict(last=-1)) == B.SKVQ_ERR_INVALID_ARG
    assert weights(lib, rope=(None, 64, 0, 8)) == B.SKVQ_ERR_INVALID_ARG and weights(lib, rope=(FAKE + 8, 64, 0, 8)) == B.SKVQ_ERR_MISALIGNED
    # nothing new and the weights in place: nothing to do
    assert weights(lib, batch=dict(n_tokens=0), q=None, lse=None, args=dict(workspace=None)) == B.SKVQ_OK
    assert weights(lib, batch=dict(max_new=0), q=None, lse=None, args=dict(workspace=None)) == B.SKVQ_OK
    cfg, pool, batch = structs()
    assert lib.skvq_paged_weights(ctypes.byref(cfg), ctypes.byref(pool), ctypes.byref(batch), None, FAKE, 1024, FAKE, None, None) == B.SKVQ_ERR_INVALID_ARG


def test_evict_refusals(lib):
    for bad in (dict(keep=0), dict(first=-1), dict(recent=-1), dict(recent=127), dict(first=73), dict(first=2**31 - 1), dict(weights=None), dict(lens_out=None),
                dict(kept=None), dict(page_table_out=FAKE, max_pages_out=0)):
        assert evict(lib, args=bad) == B.SKVQ_ERR_INVALID_ARG, bad
    for name in ("page_table_out", "slots_out", "lens_out", "ring_from_out", "kept"):
        assert evict(lib, args={name: FAKE + 2, "max_pages_out": 9}) == B.SKVQ_ERR_MISALIGNED, name
    assert evict(lib, args=dict(page_table_out=FAKE, max_pages_out=3)) == B.SKVQ_ERR_CAPACITY       # 200 tokens need four pages of 64
    assert evict(lib, cfg=dict(window=8193, ring_tokens=8193), args=dict(recent=8193, keep=9000)) == B.SKVQ_ERR_UNSUPPORTED
    cfg, pool, batch = structs()
    call = lib.skvq_paged_evict
    assert call(ctypes.byref(cfg), ctypes.byref(pool), ctypes.byref(batch), None, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(ctypes.byref(cfg), ctypes.byref(pool), None, None, None) == B.SKVQ_ERR_INVALID_ARG


def test_workspace_sizes(lib):
    cfg, _, batch = structs(batch=dict(n_tokens=70, max_new=40))
    assert B.skvq_paged_evict_workspace_size(cfg, batch) > 0
    for bad in (dict(n_seqs=0), dict(n_seqs=2049)):
        assert B.skvq_paged_evict_workspace_size(cfg, structs(batch=bad)[2]) == 0
        assert B.skvq_paged_weights_workspace_size(cfg, structs(batch=bad)[2]) == 0
    one = B.skvq_paged_weights_workspace_size(cfg, batch)
    assert one > 0
    for bad in (dict(n_tokens=0), dict(max_new=0), dict(max_len=-1), dict(max_new=1 << 30)):
        assert B.skvq_paged_weights_workspace_size(cfg, structs(batch=bad)[2]) == 0, bad
    assert B.skvq_paged_weights_workspace_size(cfg, batch, -1) == 0
    # 64 prompts of 4096 tokens judged by their last 32 need a fraction of what all their queries need
    many = structs(batch=dict(n_seqs=4, n_tokens=4 * 4096, max_new=4096, max_len=4096, max_pages=64))[2]
    assert B.skvq_paged_weights_workspace_size(cfg, many, 32) * 50 < B.skvq_paged_weights_workspace_size(cfg, many, 0)
    # and never more than the rows of the step, padded, however ragged it is
    ragged = structs(batch=dict(n_seqs=100, slots=FAKE, n_tokens=5000, max_new=4000, max_len=4096, max_pages=64))[2]
    assert B.skvq_paged_weights_workspace_size(cfg, ragged, 0) <= (5000 * 4 + 100 * 128) * 2 * (128 * 2 + 16) * 2


def test_python_checks(lib):
    """The binding's own checks, on the CPU: a cache cannot be made here, so its methods are called on a stand-in."""
    class Stand(B.SkvqPagedCache):
        def __init__(self):
            self.cfg, self.index = structs()[0], -1
    c = Stand()
    for bad in (torch.zeros(4, 2, 8, dtype=torch.float64), torch.zeros(3, 2, 8), torch.zeros(4, 3, 8), torch.zeros(4, 8), torch.zeros(4, 2, 16)[:, :, ::2]):
        with pytest.raises(AssertionError):
            c._weights(bad)
    assert c._weights(torch.zeros(4, 2, 9)) == 9
