"""Eviction: what skipped sequences keep."""
import pytest
import torch

import test_gpu_rope_paged as base
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


def words(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("aliased", [False, True])
def test_a_skipped_sequence_keeps_its_ring_from(aliased):
    p = base.Paged(n_seqs=5, seed=7, slots=[0, 1, 2, 3, 4], P=16)
    p.append([100] * 5)
    lens, first = words(100, 401, 100, -1, 100), words(61, 77, 500, 9, -3)
    p.slots[2] = 5      # no such slot
    batch = p.cache.batch(p.page_table, lens, words(*[0] * 6), 0, 0, 400, slots=p.slots, ring_from=first)
    out = first if aliased else torch.full_like(first, 99)
    kept, lens_out, ring_from = p.cache.evict(batch, torch.rand(5, 2, 400, device="cuda"), 50, 0, 40, ring_from_out=out)
    assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_BATCH and ring_from is out
    assert lens_out.tolist() == [50, 401, 100, -1, 50] and (kept[1:4] == -1).all()
    R = p.cache.cfg.ring_tokens
    begin = 100 - min(R, 40)
    assert out.tolist() == [max(begin, 61) - 50, 77, 500, 9, begin - 50]
