"""Eviction: what skipped sequences keep, and rings wider than an eviction moves."""
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


def test_rows_of_a_wide_ring_that_stay_where_they_are_still_count():
    """8192 ring rows are moved at most; of a sequence that keeps its slot, and whose numbers shift by whole turns of the ring or not at all,
    every row is in its place without a move."""
    H, D, P, R, recent, keep = 1, 64, 256, 9000, 8500, 9100
    lens = [8900, R + keep, keep + 900, 8900]
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = -(-max(lens) // P)
    cache = B.SkvqPagedCache(H, H, D, 64, 16, P, 4 * pages, 5, ring_tokens=R)
    for name in ("k_win", "v_win"):
        getattr(cache, name).copy_(torch.randn(getattr(cache, name).shape, generator=g, device="cuda"))
    before = [cache.k_win.clone(), cache.v_win.clone()]
    table = torch.arange(4 * pages, dtype=torch.int32, device="cuda").view(4, pages)
    batch = cache.batch(table, words(*lens), words(*[0] * 5), 0, 0, max(lens), slots=words(0, 1, 2, 3))
    w = torch.rand(5, H, max(lens), generator=g, device="cuda")
    _, lens_out, ring_from = cache.evict(batch, w, keep, 0, recent, slots_out=words(0, 1, 2, 4))
    assert lens_out.tolist() == [8900, keep, keep, 8900]
    # whole, in place: the ring holds all of it; shifted by one turn: the recent ones; shifted otherwise, or in another slot: the rows that were moved
    assert ring_from.tolist() == [0, keep - recent, keep - 8192, 8900 - 8192]
    for x, y in zip(before, (cache.k_win, cache.v_win)):
        assert torch.equal(y[:2], x[:2]) and torch.equal(y[3], x[3])
        for b, to, gone in ((2, 2, 900), (3, 4, 0)):
            t = torch.arange(int(ring_from[b]), int(lens_out[b]), device="cuda")
            assert torch.equal(y[to][:, t % R], x[b][:, (t + gone) % R])
    assert int(cache.status[0]) == 0
