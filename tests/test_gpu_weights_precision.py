"""Accumulated attention weights on inputs whose errors add up: keys off the fp16 grid to one side, queries whose small entries use all their
bits, small keys under large queries.  Bounds: precision_reference."""
import math

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


def weights_of(codes, meta, q, lse, sm_scale):
    """One KV head, every query a token's: float64 [n]."""
    n, D = codes.shape
    rows, G, P = q.shape[0], D // meta.shape[1], 16
    pages = -(-n // P)
    cache = B.SkvqPagedCache(1, 1, D, G, 0, P, pages, 1)
    padded = torch.zeros(pages * P, D, dtype=torch.uint8)
    padded[:n] = codes
    cache.k_codes.copy_((padded[:, 0::2] | padded[:, 1::2] << 4).view(pages, 1, P, D // 2))
    cache.k_meta.view(-1, D // G, 2)[:n] = meta.cuda()
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    batch = cache.batch(torch.arange(pages, dtype=torch.int32, device="cuda")[None], dev([n]), dev([0, rows]), rows, rows, n)
    w = cache.new_weights(n)
    cache.accumulate_weights(batch, q[:, None].contiguous().cuda(), lse[:, None].contiguous().cuda(), None, sm_scale, out=w, causal=False)
    assert int(cache.status[0]) == 0
    return w[0, 0].cpu().double()


def ratio(codes, meta, q, errors, top):
    """The largest ratio of error to allowed error."""
    exact = q.double() @ plain.keys(codes, meta).t()
    sm_scale = plain.scale_for(exact, top)
    lse = (sm_scale * exact).amax(-1).float()
    want, allowed = plain.weights(exact, errors, lse, sm_scale)
    return float(((weights_of(codes, meta, q, lse, sm_scale) - want).abs() / allowed).max())


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


@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("rows", [24, 200])
def test_scores_of_many_rows_are_not_too_small_on_average(G, rows):
    """Sums cut toward zero make every score too small.  The scale is the fp32 number that comes nearest to making up for it: within half a
    step of its own, and 0.15 of 2^-24 for the measured share that it goes by."""
    g, D, n = torch.Generator().manual_seed(G + rows), 128, 4096
    codes = torch.randint(0, 16, (n, D), generator=g).to(torch.uint8)
    meta = torch.tensor([0.125, -0.9375], dtype=torch.float16).expand(n, D // G, 2)
    q = torch.randn(rows, D, generator=g).half()
    sm_scale = float(torch.tensor(D ** -0.5))
    share, offs = 2.0 ** -24 * (1 / (sm_scale * 16) + 0.15), []
    for r in range(8):      # a row at a time, both signs; the others add nothing
        for sign in (1, -1):
            s = sign * sm_scale * (q[r].double() @ plain.keys(codes, meta).t())
            lse = torch.full((rows,), math.inf)
            lse[r] = s.max().float()
            got = torch.log(weights_of(codes, meta, sign * q, lse, sm_scale)) + lse[r].double()
            near = (s > lse[r].double() - 2) & (s > 1)
            offs.append(((got - s) / s)[near])
    offs = torch.cat(offs)
    assert len(offs) > 200 and abs(float(offs.mean())) <= share, float(offs.mean()) * 2.0 ** 24
