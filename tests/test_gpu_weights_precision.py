"""Accumulated attention weights on inputs whose errors add up: keys off the fp16 grid to one side, queries whose small entries use all their
bits, small keys under large queries.  Bounds: precision_reference."""
import pytest
import torch

import precision_reference as plain
from paper_2405_06219_b200 import binding as B
from paper_2405_06219_b200 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build_library()
    B.lib()


def ratio(codes, meta, q, errors, top):
    """One KV head, every query a query head's or a token's; the largest ratio of error to allowed error."""
    n, D = codes.shape
    rows, G, P = q.shape[0], D // meta.shape[1], 16
    pages = -(-n // P)
    cache = B.SkvqPagedCache(1, 1, D, G, 0, P, pages, 1)
    padded = torch.zeros(pages * P, D, dtype=torch.uint8)
    padded[:n] = codes
    cache.k_codes.copy_((padded[:, 0::2] | padded[:, 1::2] << 4).view(pages, 1, P, D // 2))
    cache.k_meta.view(-1, D // G, 2)[:n] = meta.cuda()
    exact = q.double() @ plain.keys(codes, meta).t()
    sm_scale = plain.scale_for(exact, top)
    lse = (sm_scale * exact).amax(-1).float()
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    batch = cache.batch(torch.arange(pages, dtype=torch.int32, device="cuda")[None], dev([n]), dev([0, rows]), rows, rows, n)
    w = cache.new_weights(n)
    cache.accumulate_weights(batch, q[:, None].contiguous().cuda(), lse[:, None].contiguous().cuda(), None, sm_scale, out=w, causal=False)
    assert int(cache.status[0]) == 0
    want, allowed = plain.weights(exact, errors, lse, sm_scale)
    return float(((w[0, 0].cpu().double() - want).abs() / allowed).max())


@pytest.mark.parametrize("D,G", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("rows", [1, 4, 7, 16])
def test_small_entries_of_queries_count_with_all_their_bits(D, G, rows):
    g = torch.Generator().manual_seed(D * G + rows)
    codes = torch.randint(0, 16, (77, D), generator=g).to(torch.uint8)
    meta = torch.tensor([0.25, 0.0], dtype=torch.float16).expand(77, D // G, 2)
    q = plain.queries_with_tails(rows, D, g)
    assert ratio(codes, meta, q, plain.few_error(codes, meta, q, plain.TAIL), 16.0) <= 1


@pytest.mark.parametrize("D,G", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("rows", [1, 3, 8, 16, 17, 130])
def test_keys_are_not_rounded_to_fp16(D, G, rows):
    g = torch.Generator().manual_seed(D + G + rows)
    codes, meta = plain.rounded_one_way(77, D, G, 1.0, g)
    q = (torch.rand(rows, D, generator=g) + 0.25).half()
    errors = (plain.few_error if rows <= 16 else plain.many_error)(codes, meta, q)
    assert ratio(codes, meta, q, errors, 16.0) <= 1


@pytest.mark.parametrize("D,G", [(128, 32), (128, 128), (64, 64)])
@pytest.mark.parametrize("rows", [1, 8, 40])
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4])
def test_small_keys_under_large_queries(D, G, rows, size):
    g = torch.Generator().manual_seed(D + G + rows)
    h, z = torch.rand(77, D // G, generator=g) * size, torch.randn(77, D // G, generator=g) * 8 * size
    codes, meta = torch.randint(0, 16, (77, D), generator=g).to(torch.uint8), torch.stack((h, z), -1).half()
    q = (torch.rand(rows, D, generator=g) + 0.25).half() * 500
    errors = (plain.few_error if rows <= 16 else plain.many_error)(codes, meta, q)
    assert ratio(codes, meta, q, errors, 16.0) <= 1
