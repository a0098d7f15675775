"""Layer norm's gradient over many rows, by sums that are exact in any order: every row counts once, in every kernel, wherever the
tensors start and whatever the weights' type."""
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .buffers import Buffer

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def whole_case(rows, dim):
    """Whole numbers with mu = 0 and r = 1, weights that are powers of two: sums over the rows stay below 2^24 and are exact."""
    gen = torch.Generator().manual_seed(rows + 31 * dim)
    x, dy = (torch.randint(-8, 9, (rows, dim), generator=gen).float() for _ in range(2))
    weight = 2.0 ** torch.randint(-2, 3, (dim,), generator=gen).float()
    assert (x * dy).abs().sum(0).max() < 2 ** 24 and dy.abs().sum(0).max() < 2 ** 24
    return x, dy, weight


def run(x, dy, weight, kinds, shift, w_type, keep=(True, True, True)):
    rows, dim = x.shape
    bx, bdy = Buffer(rows * dim, kinds[0], shift, x.view(-1).to(kinds[0])), Buffer(rows * dim, kinds[1], shift, dy.view(-1).to(kinds[1]))
    bs = Buffer(2 * rows, F32, shift, torch.tensor([0.0, 1.0]).repeat(rows))
    w = None if weight is None else Buffer(dim, w_type, shift, weight.to(w_type))
    out = [Buffer(n, t, shift) if k else None for n, t, k in zip((rows * dim, dim, dim), (kinds[0], F32, F32), keep)]
    sums = keep[1] or keep[2]
    work = Buffer(mqg.mqg_layer_norm_workspace_floats(rows, dim), F32, 0) if sums else None
    mqg.mqg_layer_norm_grad(bdy.view, bx.view, rows, dim, None if w is None else w.view, bs.view,
                            *[None if b is None else b.view for b in out], None if work is None else work.view)
    if work is not None:
        work.check()
    return [None if b is None else b.cpu() for b in out]


def dx_close(dx, x, dy, weight, kind):
    a = dy.double() * (1.0 if weight is None else weight.double())
    x = x.double()
    m1, m2 = a.mean(1, keepdim=True), (a * x).mean(1, keepdim=True)
    want = a - m1 - x * m2
    # the row's two sums: 44 additions in a chain at most, mean, the two products and sums of the result
    off = 2.0 ** -24 * (5 * a.abs() + 50 * a.abs().mean(1, keepdim=True) + 54 * x.abs() * (a * x).abs().mean(1, keepdim=True))
    half = 2.0 ** -24 if kind == F32 else 2.0 ** -8
    got = dx.double().view(want.shape)
    assert ((got - want).abs() <= off * (1 + half) + half * want.abs() + 1e-40).all()


# many turns of short rows, of long ones, pairs of CTAs, columns by a kernel of their own
TALL = [(70_001, 16), (70_001, 33), (70_001, 64), (131_072, 8), (200_003, 3), (40_003, 264), (30_001, 385), (9_001, 768), (16_411, 515), (3_001, 2056),
        (3_001, 2050), (1_999, 4100), (1_501, 4099), (1_303, 8192), (1_301, 5003), (1_500, 9001), (1_500, 12_288), (901, 12_287), (700, 16_380),
        (600, 14_000), (333, 16_400), (331, 17_001)]


@pytest.mark.parametrize("kinds", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("rows,dim", TALL)
def test_every_row_of_many_is_counted_once(rows, dim, kinds):
    x, dy, weight = whole_case(rows, dim)
    _, dw, db = run(x, dy, weight, kinds, 0, F32)
    assert torch.equal(dw, (x * dy).sum(0)) and torch.equal(db, dy.sum(0))


# several turns off the boundaries of a vector, weights in either type
@pytest.mark.parametrize("shift,w_type", [(1, BF16), (2, F32), (3, BF16), (4, BF16), (8, BF16)])
@pytest.mark.parametrize("kinds", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("rows,dim", [(20_011, 64), (9_001, 264), (5_003, 516), (4_001, 1028), (2_003, 2056), (701, 4104), (401, 8192), (700, 12_288), (301, 9001)])
def test_several_turns_wherever_the_tensors_start(rows, dim, kinds, shift, w_type):
    x, dy, weight = whole_case(rows, dim)
    dx, dw, db = run(x, dy, weight, kinds, shift, w_type)
    assert torch.equal(dw, (x * dy).sum(0)) and torch.equal(db, dy.sum(0))
    dx_close(dx, x, dy, weight, kinds[0])


@pytest.mark.parametrize("dim", [64, 515, 1024, 4096, 9001, 12_288, 17_000])
@pytest.mark.parametrize("weighted", [False, True])
def test_the_rows_gradient_alone(dim, weighted):
    """Without the sums, a workspace and, in one form, weights: into a buffer that holds something else."""
    for kinds in ((F32, F32), (BF16, BF16), (BF16, F32)):
        x, dy, weight = whole_case(50, dim)
        weight = weight if weighted else None
        dx, dw, db = run(x, dy, weight, kinds, 0, F32, (True, False, False))
        assert dw is None and db is None
        dx_close(dx, x, dy, weight, kinds[0])


@pytest.mark.parametrize("kinds", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("rows,dim", [(20_011, 64), (9_001, 264), (5_003, 516), (4_001, 1028), (2_003, 2056), (701, 4104), (401, 8192), (300, 12_288), (301, 9001),
                                      (70, 16_400)])
def test_forward_of_several_turns_wherever_the_rows_start(rows, dim, kinds):
    """Rows of -1 and 1 in equal numbers: mu = 0, the squares' mean is 1, and y = x r w + b with one r for all."""
    even = dim // 2 * 2
    gen = torch.Generator().manual_seed(dim)
    sign = torch.ones(rows, dim)
    sign[:, torch.randperm(even, generator=gen)[:even // 2]] = -1.0
    if dim != even:
        sign[:, -1] = 0.0
    weight, bias = 2.0 ** torch.randint(-2, 3, (dim,), generator=gen).float(), torch.randint(-3, 4, (dim,), generator=gen).float()
    r = (even / dim + 1e-5) ** -0.5
    want = sign.double() * r * weight.double() + bias.double()
    for shift, w_type in ((1, BF16), (2, F32), (4, BF16)):
        x, y = Buffer(rows * dim, kinds[0], shift, sign.view(-1).to(kinds[0])), Buffer(rows * dim, kinds[1], shift)
        w, b = (Buffer(dim, w_type, shift, t.to(w_type)) for t in (weight, bias))
        stats = Buffer(2 * rows, F32, shift)
        mqg.mqg_layer_norm(x.view, rows, dim, w.view, b.view, 1e-5, y.view, stats.view)
        got, half = y.cpu().double().view(rows, dim), 2.0 ** -24 if kinds[1] == F32 else 2.0 ** -8
        # sums of whole numbers are exact; the mean of the squares, eps, its sum, the root (halved), the reciprocal; two products and a sum
        off = 2.0 ** -24 * (6 * (want - bias.double()).abs() + want.abs())
        assert ((got - want).abs() <= off * (1 + half) + half * want.abs()).all()
        s = stats.cpu().view(rows, 2).double()
        assert not s[:, 0].any() and ((s[:, 1] - r).abs() <= 4 * 2.0 ** -24 * r).all()
