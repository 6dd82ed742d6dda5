"""Sizing and refusals of the paged and rotary calls at the ends of their ranges: host only, nothing is launched."""
import ctypes

import pytest

import test_rope_paged_host as base
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build

FAKE = 0x1000


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
