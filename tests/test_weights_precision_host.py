"""What tests/test_gpu_weights_precision.py can tell apart: forms that lose bits are outside its bounds, those that keep them inside (CPU)."""
import pytest
import torch

import precision_reference as plain


def off(scores, codes, meta, q, errors, top):
    """The largest ratio of error to allowed error of weights from `scores`."""
    exact = q.double() @ plain.keys(codes, meta).t()
    sm_scale = plain.scale_for(exact, top)
    lse = (sm_scale * exact).amax(-1).float()
    want, allowed = plain.weights(exact, errors, lse, sm_scale)
    got = torch.exp(sm_scale * scores - lse.double()[:, None]).sum(0)
    return float(((got - want).abs() / allowed).max())


@pytest.mark.parametrize("D,G", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("rows", [17, 130])
def test_keys_rounded_to_fp16_are_noticed(D, G, rows):
    g = torch.Generator().manual_seed(D + G + rows)
    codes, meta = plain.rounded_one_way(50, D, G, 1.0, g)
    q = (torch.rand(rows, D, generator=g) + 0.25).half()
    K, errors = plain.keys(codes, meta), plain.many_error(codes, meta, q)
    assert off(q.double() @ K.half().double().t(), codes, meta, q, errors, 16.0) > 2
    assert off(q.double() @ plain.two_parts(K).t(), codes, meta, q, errors, 16.0) < 1


@pytest.mark.parametrize("D,G", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
def test_products_cut_at_subnormal_codes_are_noticed(D, G):
    """A code as c 2^-24 is aligned as if it were 1024: products cut at 2^-15 of the largest query."""
    g = torch.Generator().manual_seed(D * G)
    codes = torch.randint(0, 16, (50, D), generator=g).to(torch.uint8)
    meta = torch.tensor([0.25, 0.0], dtype=torch.float16).expand(50, D // G, 2)
    q = plain.queries_with_tails(4, D, g)
    errors = plain.few_error(codes, meta, q, plain.TAIL)
    assert off(plain.cut_products(codes, meta, q, 1024 * plain.FINE), codes, meta, q, errors, 16.0) > 2
    assert off(plain.cut_products(codes, meta, q, 256 * plain.FINE), codes, meta, q, errors, 16.0) < 1


def test_two_fp16_parts_hold_a_key_whatever_its_size():
    """Parameters are multiples of 2^-24, so is a key, and so are both its parts: nothing is lost at fp16's lower end."""
    g = torch.Generator().manual_seed(1)
    for size in (1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.1, 1.0, 10.0, 1000.0, 3000.0):
        h, z = (torch.rand(20000, generator=g) * size).half(), (torch.randn(20000, generator=g) * 8 * size).half()
        for c in range(16):
            x = h.double() * c + z.double()
            x = x[x.abs() <= 65440]      # what a key may be
            assert ((plain.two_parts(x) - x).abs() <= x.abs() * 2.0 ** -22).all(), (size, c)
