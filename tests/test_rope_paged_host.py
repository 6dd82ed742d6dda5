"""Rotary frequencies and the refusals of the paged calls: host only, nothing is launched."""
import ctypes
import math

import pytest

from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.lib()


# ------------------------------------------------------------------------------------------------ frequencies
def scaling(kind=0, base=10000.0, factor=4.0, original=4096, fast=32.0, slow=1.0):
    return B.SkvqRopeScaling(kind, original, base, factor, fast, slow)


@pytest.mark.parametrize("rot", [2, 64, 128, 256])
def test_frequencies_follow_their_formulas(lib, rot):
    plain, a = B.skvq_rope_frequencies(rot, scaling(B.SKVQ_ROPE_PLAIN))
    assert a == 1.0 and plain == pytest.approx([10000.0 ** (-2 * j / rot) for j in range(rot // 2)], rel=1e-14)
    linear, a = B.skvq_rope_frequencies(rot, scaling(B.SKVQ_ROPE_LINEAR))
    assert a == 1.0 and linear == pytest.approx([f / 4 for f in plain], rel=1e-14)
    if rot > 2:
        ntk, a = B.skvq_rope_frequencies(rot, scaling(B.SKVQ_ROPE_NTK))
        base = 10000.0 * 4.0 ** (rot / (rot - 2))
        assert a == 1.0 and ntk == pytest.approx([base ** (-2 * j / rot) for j in range(rot // 2)], rel=1e-13)
        # the fastest pair keeps its frequency, the slowest is divided by the factor
        assert ntk[0] == 1.0 and ntk[-1] == pytest.approx(plain[-1] / 4, rel=1e-12)
    yarn, a = B.skvq_rope_frequencies(rot, scaling(B.SKVQ_ROPE_YARN))
    assert a == pytest.approx(0.1 * math.log(4.0) + 1.0, rel=1e-15)
    for f, y in zip(plain, yarn):
        turns = 4096 * f / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
        assert y == pytest.approx(keep * f + (1 - keep) * f / 4, rel=1e-13)
    assert yarn[0] == plain[0]


@pytest.mark.parametrize("kw,rot,code", [
    (dict(), 3, B.SKVQ_ERR_INVALID_ARG), (dict(), 0, B.SKVQ_ERR_INVALID_ARG), (dict(), 258, B.SKVQ_ERR_UNSUPPORTED),
    (dict(kind=4), 64, B.SKVQ_ERR_UNSUPPORTED), (dict(kind=-1), 64, B.SKVQ_ERR_UNSUPPORTED), (dict(base=1.0), 64, B.SKVQ_ERR_INVALID_ARG),
    (dict(base=math.nan), 64, B.SKVQ_ERR_INVALID_ARG), (dict(kind=1, factor=0.5), 64, B.SKVQ_ERR_INVALID_ARG),
    (dict(kind=1, factor=math.inf), 64, B.SKVQ_ERR_INVALID_ARG), (dict(kind=2), 2, B.SKVQ_ERR_UNSUPPORTED),
    (dict(kind=3, original=0), 64, B.SKVQ_ERR_INVALID_ARG), (dict(kind=3, fast=1.0), 64, B.SKVQ_ERR_INVALID_ARG),
    (dict(kind=3, slow=-1.0), 64, B.SKVQ_ERR_INVALID_ARG),
])
def test_frequency_refusals(lib, kw, rot, code):
    with pytest.raises(B.SkvqError) as e:
        B.skvq_rope_frequencies(rot, scaling(**kw))
    assert e.value.code == code


def test_table_refusals(lib):
    f = (ctypes.c_double * 200)(*[0.5] * 200)
    call = lib.skvq_rope_table
    assert call(None, 1, 1.0, 0, 1, 16, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(f, 0, 1.0, 0, 1, 16, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(f, 129, 1.0, 0, 1, 16, None) == B.SKVQ_ERR_UNSUPPORTED
    assert call(f, 4, math.nan, 0, 1, 16, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(f, 4, 1.0, -1, 1, 16, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(f, 4, 1.0, 1 << 31, 1, 16, None) == B.SKVQ_ERR_UNSUPPORTED
    assert call(f, 4, 1.0, 0, -1, 16, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(f, 4, 1.0, 0, 1, None, None) == B.SKVQ_ERR_INVALID_ARG
    assert call(f, 4, 1.0, 0, 1, 20, None) == B.SKVQ_ERR_MISALIGNED
    assert call(f, 4, 1.0, 0, 0, None, None) == B.SKVQ_OK
    f[2] = math.inf
    assert call(f, 4, 1.0, 0, 1, 16, None) == B.SKVQ_ERR_INVALID_ARG


def test_rotation_refusals(lib):
    before = B.skvq_launch_count()
    fake = 0x1000

    def call(rope=(fake, 64, 0, 8), dtype=B.SKVQ_F16, D=128, a=(fake, fake, 1024, 128, 1024, 128, 8), b=None, pos=fake, T=4, inv=0, status=None):
        r = B.SkvqRope(*rope)
        ta = None if a is None else ctypes.byref(B.SkvqRopeTensor(*a))
        tb = None if b is None else ctypes.byref(B.SkvqRopeTensor(*b))
        return lib.skvq_rope_apply(ctypes.byref(r), dtype, D, ta, tb, pos, T, inv, status, None)

    assert call(a=None) == B.SKVQ_ERR_INVALID_ARG
    assert call(T=-1) == B.SKVQ_ERR_INVALID_ARG
    assert call(inv=2) == B.SKVQ_ERR_INVALID_ARG
    assert call(dtype=3) == B.SKVQ_ERR_UNSUPPORTED
    assert call(D=0) == B.SKVQ_ERR_INVALID_ARG
    assert call(D=520) == B.SKVQ_ERR_UNSUPPORTED
    assert call(rope=(fake, 130, 0, 8)) == B.SKVQ_ERR_INVALID_ARG       # more than the head
    assert call(rope=(fake, 63, 0, 8)) == B.SKVQ_ERR_INVALID_ARG        # odd
    assert call(rope=(fake, 64, 2, 8)) == B.SKVQ_ERR_INVALID_ARG
    assert call(rope=(None, 64, 0, 8)) == B.SKVQ_ERR_INVALID_ARG
    assert call(rope=(fake + 4, 64, 0, 8)) == B.SKVQ_ERR_MISALIGNED
    assert call(pos=None) == B.SKVQ_ERR_INVALID_ARG
    assert call(pos=fake + 2) == B.SKVQ_ERR_MISALIGNED
    assert call(status=fake + 1) == B.SKVQ_ERR_MISALIGNED
    assert call(a=(fake + 1, fake, 1024, 128, 1024, 128, 8)) == B.SKVQ_ERR_MISALIGNED
    assert call(a=(fake, None, 1024, 128, 1024, 128, 8)) == B.SKVQ_ERR_INVALID_ARG
    assert call(a=(fake, fake, 1024, 128, 1024, 128, -1)) == B.SKVQ_ERR_INVALID_ARG
    assert call(b=(None, fake, 1024, 128, 1024, 128, 8)) == B.SKVQ_ERR_INVALID_ARG
    assert call(T=0) == B.SKVQ_OK
    assert call(a=(None, None, 0, 0, 0, 0, 0)) == B.SKVQ_OK             # no heads: nothing to do
    assert B.skvq_launch_count() == before


# ------------------------------------------------------------------------------------------------ the paged cache
def pcfg(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, group_size=64, window=128, ring_tokens=128, page_tokens=64, n_pages=10,
                n_slots=4, dtype=B.SKVQ_F16)
    base.update(kw)
    return B.SkvqPagedConfig(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(), B.SKVQ_OK), (dict(head_dim=64), B.SKVQ_OK), (dict(head_dim=96), B.SKVQ_ERR_UNSUPPORTED),
    (dict(head_dim=64, group_size=128), B.SKVQ_ERR_UNSUPPORTED), (dict(group_size=16), B.SKVQ_ERR_UNSUPPORTED),
    (dict(page_tokens=8), B.SKVQ_ERR_UNSUPPORTED), (dict(page_tokens=48), B.SKVQ_ERR_UNSUPPORTED), (dict(page_tokens=256), B.SKVQ_OK),
    (dict(n_q_heads=7), B.SKVQ_ERR_UNSUPPORTED), (dict(n_q_heads=32), B.SKVQ_OK), (dict(n_q_heads=34), B.SKVQ_ERR_UNSUPPORTED),
    (dict(window=-1), B.SKVQ_ERR_INVALID_ARG), (dict(ring_tokens=127), B.SKVQ_ERR_INVALID_ARG), (dict(window=0, ring_tokens=0), B.SKVQ_OK),
    (dict(n_pages=0), B.SKVQ_ERR_INVALID_ARG), (dict(n_slots=0), B.SKVQ_ERR_INVALID_ARG), (dict(dtype=B.SKVQ_F32), B.SKVQ_ERR_UNSUPPORTED),
    (dict(dtype=B.SKVQ_BF16), B.SKVQ_OK), (dict(n_kv_heads=0), B.SKVQ_ERR_INVALID_ARG),
])
def test_paged_config_validation(lib, kw, code):
    assert B.skvq_check_paged_config(pcfg(**kw)) == code
    assert lib.skvq_check_paged_config(None) == B.SKVQ_ERR_INVALID_ARG


def test_paged_sizes_follow_the_documented_layout(lib):
    rows = 10 * 2 * 64
    assert B.skvq_paged_cache_sizes(pcfg()) == [rows * 64] * 2 + [rows * 2 * 4] * 2 + [4 * 2 * 128 * 128 * 2] * 2
    assert B.skvq_paged_cache_sizes(pcfg(head_dim=64, group_size=32, window=0, ring_tokens=64)) == [rows * 32] * 2 + [rows * 2 * 4] * 2 + [0, 0]


def test_paged_calls_refuse_bad_arguments_before_any_launch(lib):
    fake = 0x1000
    before = B.skvq_launch_count()

    def call(which="append", cfg=None, pool=None, batch=None, rope=None, x=fake, stride=1024, y=fake, ystride=1024, args=None, window=0, lse=None):
        c = ctypes.byref(pcfg(**(cfg or {})))
        fields = dict(k_codes=fake, v_codes=fake, k_meta=fake, v_meta=fake, k_win=fake, v_win=fake)
        fields.update(pool or {})
        p = ctypes.byref(B.SkvqPagedCacheStruct(**fields))
        fields = dict(page_table=fake, lens=fake, starts=fake, slots=None, n_seqs=3, max_pages=5, n_tokens=7, max_new=4, max_len=320)
        fields.update(batch or {})
        b = ctypes.byref(B.SkvqPagedBatch(**fields))
        r = None if rope is None else ctypes.byref(B.SkvqRope(*rope))
        if which == "append":
            return lib.skvq_paged_append(c, p, b, r, x, y, stride, ystride, None)
        if which == "read":
            return lib.skvq_paged_read(c, p, b, window, x, y, stride, ystride, None)
        fields = dict(sm_scale=0.1, causal=1, n_splits=0, workspace=fake, workspace_bytes=1 << 40)
        fields.update(args or {})
        return lib.skvq_paged_attention(c, p, b, r, x, stride, y, ystride, lse, ctypes.byref(B.SkvqPagedAttnArgs(**fields)), None)

    for which in ("append", "read", "attention"):
        assert call(which, cfg=dict(head_dim=80)) == B.SKVQ_ERR_UNSUPPORTED
        for name in ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win"):
            assert call(which, pool={name: None}) == B.SKVQ_ERR_INVALID_ARG, name
            assert call(which, pool={name: fake + 8}) == B.SKVQ_ERR_MISALIGNED, name
        for name in ("page_table", "lens", "starts"):
            assert call(which, batch={name: None}) == B.SKVQ_ERR_INVALID_ARG, name
            assert call(which, batch={name: fake + 2}) == B.SKVQ_ERR_MISALIGNED, name
        assert call(which, batch=dict(n_seqs=0)) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, batch=dict(n_seqs=2049, slots=fake)) == B.SKVQ_ERR_UNSUPPORTED
        assert call(which, batch=dict(n_seqs=5)) == B.SKVQ_ERR_CAPACITY             # four ring slots and no slot numbers
        assert call(which, batch=dict(max_len=321)) == B.SKVQ_ERR_CAPACITY          # five pages of 64
        assert call(which, batch=dict(max_new=-1)) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, batch=dict(n_tokens=-1)) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, batch=dict(max_new=1 << 30)) == B.SKVQ_ERR_UNSUPPORTED
        assert call(which, x=fake + 2) == B.SKVQ_ERR_MISALIGNED
        assert call(which, stride=1028) == B.SKVQ_ERR_MISALIGNED
        assert call(which, stride=128) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, batch=dict(n_tokens=0)) == B.SKVQ_OK and call(which, batch=dict(max_new=0)) == B.SKVQ_OK
    for which in ("append", "attention"):
        assert call(which, x=None) == B.SKVQ_ERR_INVALID_ARG and call(which, y=None) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, rope=(None, 64, 0, 8)) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, rope=(fake, 130, 0, 8)) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, rope=(fake, 7, 0, 8)) == B.SKVQ_ERR_INVALID_ARG
        assert call(which, rope=(fake + 8, 64, 0, 8)) == B.SKVQ_ERR_MISALIGNED
    assert call("read", window=2) == B.SKVQ_ERR_INVALID_ARG
    assert call("read", x=None, y=None) == B.SKVQ_OK
    assert call("attention", args=dict(causal=2)) == B.SKVQ_ERR_INVALID_ARG
    assert call("attention", args=dict(n_splits=-1)) == B.SKVQ_ERR_INVALID_ARG
    assert call("attention", args=dict(workspace=None, n_splits=2)) == B.SKVQ_ERR_WORKSPACE
    assert call("attention", args=dict(workspace_bytes=64, n_splits=2)) == B.SKVQ_ERR_WORKSPACE
    long = dict(max_pages=100, max_len=6400)      # (contexts as short as the others' here need no workspace)
    assert call("attention", batch=long, args=dict(workspace=None)) == B.SKVQ_ERR_WORKSPACE
    assert call("attention", args=dict(workspace=fake + 4)) == B.SKVQ_ERR_MISALIGNED
    assert call("attention", lse=fake + 2) == B.SKVQ_ERR_MISALIGNED
    assert B.skvq_launch_count() == before
