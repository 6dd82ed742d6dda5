"""Scratch sizes of skvq_paged_weights (CPU)."""
import pytest

from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


def size(last, n_seqs, n_tokens, max_new, max_len=8192, heads=(32, 32), D=128):
    cfg = B.SkvqPagedConfig(n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=D, group_size=64, window=0, ring_tokens=0, page_tokens=64, n_pages=10, n_slots=n_seqs,
                            dtype=B.SKVQ_F16)
    batch = B.SkvqPagedBatch(page_table=0x1000, lens=0x1000, starts=0x1000, slots=None, n_seqs=n_seqs, max_pages=-(-max_len // 64), n_tokens=n_tokens, max_new=max_new,
                             max_len=max_len)
    return B.skvq_paged_weights_workspace_size(cfg, batch, last)


@pytest.mark.parametrize("n_seqs,n_tokens,max_new", [(64, 4160, 4096), (1, 4096, 4096), (9, 20000, 4095), (2048, 5000, 2000), (3, 100, 100)])
@pytest.mark.parametrize("heads,D", [((32, 32), 128), ((32, 8), 128), ((24, 8), 64), ((32, 2), 64)])
def test_fewer_counted_tokens_need_no_more_scratch(n_seqs, n_tokens, max_new, heads, D):
    """However ragged the batch: one chunk of thousands among sequences with a token each as well."""
    most = size(0, n_seqs, n_tokens, max_new, heads=heads, D=D)
    before = 0
    for last in (1, 4, 17, 100, 500, 1023, 2048, 4095, 4096, 5000):
        now = size(last, n_seqs, n_tokens, max_new, heads=heads, D=D)
        assert before <= now <= most, last
        before = now


def test_bounds_at_their_limits():
    """The number of runs is counted from the host bounds, which may be far above what a batch holds: up to 2^63 items and more."""
    for n_seqs, heads in ((2048, (128, 128)), (2048, (65535, 65535)), (1024, (256, 256))):
        small, large = (size(0, n_seqs, 1 << 20, 1 << 30, max_len=n, heads=heads) for n in (1 << 20, 1 << 30))
        assert small == large > 0
