"""Layer norm's gradient of rows far from zero, in lengths that leave places of their threads without elements."""
import pytest
import torch

from .test_layer_norm_roundings_gpu import BF16, F32, U, gradients

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [F32, BF16], ids=str)
@pytest.mark.parametrize("rows,dim", [(3, 60), (3, 61), (5, 12), (40, 100), (700, 516), (300, 1001), (200, 1028), (40, 4100), (20, 5003), (9, 8196),
                                      (9, 9001), (700, 12_284), (5, 16_380), (5, 17_001)])
def test_rows_far_from_zero_that_do_not_fill_their_threads(rows, dim, kind):
    """x = mu = 2^121 with r = 300: mu r is beyond fp32, (x - mu) r is zero, and so dx = r (a - mean(a)), dweight = 0."""
    gen = torch.Generator().manual_seed(dim)
    dy = torch.randn(rows, dim, generator=gen).to(kind)
    weight = torch.randn(dim, generator=gen)
    x = torch.full((rows, dim), 2.0 ** 121, dtype=kind)
    stats = torch.tensor([2.0 ** 121, 300.0]).repeat(rows, 1)
    for shift in (0, 1):
        dx, dw, db = gradients(x, dy, stats, shift=shift, weight=weight)
        a = dy.double() * weight.double()
        want = 300.0 * (a - a.mean(1, keepdim=True))
        # a's rounding, the sum's 44 additions, mean, c1, the last fused product
        off = 300.0 * U * (4 * a.abs() + 50 * a.abs().mean(1, keepdim=True)) + (2.0 ** -8 if kind == BF16 else 0) * want.abs() * (1 + U)
        assert ((dx.double() - want).abs() <= off * (1 + 2.0 ** -8)).all()
        assert not dw.any() and db.isfinite().all()
