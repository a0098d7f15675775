"""Layer norm's gradient: how often sums over the rows are rounded."""
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .buffers import Buffer

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def gradients(x, dy, stats, dw_type=F32, start=None, shift=0, weight=None):
    """dx, dweight, dbias on the host; `start`: what dweight and dbias are added to."""
    rows, dim = x.shape
    bx, bdy = Buffer(rows * dim, x.dtype, shift, x.reshape(-1)), Buffer(rows * dim, dy.dtype, shift, dy.reshape(-1))
    bs, dx = Buffer(2 * rows, F32, shift, stats.reshape(-1)), Buffer(rows * dim, x.dtype, shift)
    dw, db = (Buffer(dim, dw_type, shift, start) for _ in range(2))
    w = None if weight is None else Buffer(dim, weight.dtype, shift, weight)
    work = Buffer(mqg.mqg_layer_norm_workspace_floats(rows, dim), F32, 0)
    mqg.mqg_layer_norm_grad(bdy.view, bx.view, rows, dim, None if w is None else w.view, bs.view, dx.view, dw.view, db.view, work.view,
                            add_into_grads=start is not None)
    work.check()
    return dx.cpu().view(rows, dim), dw.cpu(), db.cpu()


@pytest.mark.parametrize("dim", [8, 33, 64, 1024, 2048, 4099, 8192, 9001, 12_288, 17_000])
def test_sums_added_to_bf16_are_rounded_once(dim):
    """1 + 2^-8 lies half way between two bf16; 1 + 2^-8 + 2^-31, which fp32 does not hold, above it, and 1 - 2^-9 (1 + 2^-23) below
    half way between 1 - 2^-8 and 1."""
    sums = torch.where(torch.arange(dim) % 2 == 0, 2.0 ** -8 * (1 + 2.0 ** -23), -2.0 ** -9 * (1 + 2.0 ** -23)).float()
    dy = sums[None].clone()
    _, dw, db = gradients(torch.ones(1, dim), dy, torch.tensor([[0.0, 1.0]]), BF16, torch.ones(dim, dtype=BF16))
    want = torch.where(torch.arange(dim) % 2 == 0, 1 + 2.0 ** -7, 1 - 2.0 ** -8)
    assert torch.equal(db.float(), want) and torch.equal(dw.float(), want)


def test_sums_rounded_to_bf16_of_every_kind():
    """Ties, neighbours of ties, zeros of both signs, subnormal numbers, overflow, infinities and NaN: as one rounding from 64 bits has them."""
    start = torch.tensor([1.0, 1.0, 1.0, -1.0, -1.0, 0.0, -0.0, 3.3e38, -3.3e38, float("inf"), float("nan"), 2.0 ** -130, 0.0, 1.0, 1.0, 2.0])
    dy = torch.tensor([2.0 ** -8, 2.0 ** -8 + 2.0 ** -31, 2.0 ** -8 - 2.0 ** -32, -2.0 ** -8, -2.0 ** -8 - 2.0 ** -31, 0.0, 0.0, 3e38, -3e38, 1.0, 1.0,
                       2.0 ** -134 + 2.0 ** -149, 2.0 ** -149, 2.0 ** -60, -2.0 ** -60, 2.0 ** -40])
    want = torch.tensor([1.0, 1 + 2.0 ** -7, 1.0, -1.0, -1 - 2.0 ** -7, 0.0, 0.0, float("inf"), -float("inf"), float("inf"), float("nan"),
                         2.0 ** -130 + 2.0 ** -133, 0.0, 1.0, 1.0, 2.0])
    _, _, db = gradients(torch.ones(1, 16), dy[None], torch.tensor([[0.0, 1.0]]), BF16, start.to(BF16))
    assert torch.equal(db.float().isnan(), want.isnan()) and torch.equal(db.float().nan_to_num(9.0), want.nan_to_num(9.0)), (db, want)


# rows, elements, rows that a thread takes
SHAPES = [(512, 64, 1), (64, 64, 1), (250, 256, 2), (64, 1000, 2), (4736, 256, 1), (592, 1024, 1), (9472, 128, 1), (4736, 129, 2),
          (20_000, 33, 3), (8, 17_000, 1), (8, 16_400, 1), (300, 9001, 5)]


@pytest.mark.parametrize("rows,dim,own", SHAPES)
@pytest.mark.parametrize("kind", [F32, BF16], ids=str)
def test_sums_of_a_ctas_rows_beside_one_large_row(rows, dim, own, kind):
    """One row of 2^24 among ones, which fp32 loses where it adds them one by one.  A thread's own rows are added in fp32, 1 lost with each
    of them at most; what follows in 64 bits, with one rounding for each part and one at the end, of 1 at most each."""
    for large in (0, rows // 2, rows - 1):
        dy = torch.ones(rows, dim)
        dy[large] = 2.0 ** 24
        stats = torch.tensor([0.0, 1.0]).repeat(rows, 1)
        _, dw, db = gradients(torch.ones(rows, dim, dtype=kind), dy.to(kind), stats)
        want = 2.0 ** 24 + rows - 1
        for got in (dw, db):
            assert ((got.double() - want).abs() <= 2 * U * want + own - 1).all(), (got.double() - want).abs().max()
