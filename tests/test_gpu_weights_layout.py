"""Accumulated weights of batches that mix a chunk with single tokens, judged by their last queries: the query tiles lie one after the other."""
import pytest
import torch

from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build
from test_gpu_axes_weights_evict import Weighed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


@pytest.mark.parametrize("kw", [dict(D=128, G=64), dict(D=64, G=32, H=1, Hq=3)])
@pytest.mark.parametrize("last", [70, 139, 0])
def test_ragged_batches_with_last(kw, last):
    """The workspace of the exact size between guard regions."""
    p = Weighed(n_seqs=20, seed=last, W=16, **kw)
    new = [1, 140, 0, 1, 1, 2, 90, 1, 1, 1, 17, 1, 1, 1, 1, 1, 3, 1, 60, 1]
    p.append([40, 160] + [30] * 4 + [90] * 14)
    size = B.skvq_paged_weights_workspace_size(p.cache.cfg, p.batch(new, p.lens()), last)
    assert size <= B.skvq_paged_weights_workspace_size(p.cache.cfg, p.batch(new, p.lens()), 0)
    p.check(new, last=last)
    p.check(new, last=last, causal=False)


@pytest.mark.parametrize("rows", [1, 40])
def test_sequences_beyond_a_bound_of_no_tokens_are_reported(rows):
    p = Weighed(n_seqs=2, seed=1)
    p.append([50, 0])
    q, lse = torch.randn(2 * rows, p.Hq, p.D, device="cuda", dtype=p.dtype), torch.zeros(2 * rows, p.Hq, device="cuda")
    out = torch.full((2, p.H, 401), 7.0, device="cuda")
    p.cache.accumulate_weights(p.batch([rows, rows], [50, 0], max_len=0), q, lse, None, 0.1, out=out)
    assert int(p.cache.status[0]) == B.SKVQ_STATUS_BAD_BATCH and (out == 7).all()
