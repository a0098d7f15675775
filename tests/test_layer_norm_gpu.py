"""Layer norm and its gradient against the formulas in 64 bits."""
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .buffers import Buffer

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}                # a rounding, relative
EPS = 1e-5
U = 2.0 ** -24
# Additions that one sum over a row is off by at most: up to 32 elements of a thread one after the other, then trees over 32
# lanes and 32 warps (10), or the row's sum in 64 bits.
CHAIN = 44


def made(shape, dtype, shift, scale=1.0, mean=0.0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    n = 1
    for s in shape:
        n *= s
    b = Buffer(n, dtype, shift, (torch.randn(n, generator=gen) * scale + mean).to(dtype))
    b.shaped = b.view.view(shape)
    return b


def plain(x, w, b, eps=EPS):
    """y, mu, r, and how far fp32 may be off, all in 64 bits (a row is the last dimension)."""
    mu = x.mean(-1, keepdim=True)
    d = x - mu
    var = (d * d).mean(-1, keepdim=True)
    r = (var + eps) ** -0.5
    y = d * r * w + b
    off_mu = (CHAIN + 2) * U * x.abs().mean(-1, keepdim=True)
    # var: the sum, a square and d's own rounding twice, and the square of mu's error; r: half of that, root and reciprocal
    off_r = r * (0.5 * ((CHAIN + 5) * U + off_mu ** 2 / (var + eps)) + 3 * U)
    off_y = w.abs() * (r * off_mu + d.abs() * off_r) + 4 * U * (d * r * w).abs() + U * (y.abs() + b.abs())
    return y, mu, r, off_y, off_mu, off_r


def run(x, rows, dim, w, b, y, stats):
    mqg.mqg_layer_norm(x.view, rows, dim, None if w is None else w.view, None if b is None else b.view, EPS, y.view,
                       None if stats is None else stats.view)


def check(x, rows, dim, w, b, y, stats):
    one, zero = torch.ones(dim, dtype=torch.float64), torch.zeros(dim, dtype=torch.float64)
    want, mu, r, off_y, off_mu, off_r = plain(x.cpu().view(rows, dim).double(), one if w is None else w.cpu().double(),
                                              zero if b is None else b.cpu().double())
    got = y.cpu().view(rows, dim)
    assert ((got.double() - want).abs() <= off_y * (1 + HALF[got.dtype]) + HALF[got.dtype] * want.abs() + 1e-40).all()
    if stats is not None:
        s = stats.cpu().view(rows, 2).double()
        assert ((s[:, :1] - mu).abs() <= off_mu + 1e-40).all() and ((s[:, 1:] - r).abs() <= off_r).all()


DIMS = [1, 2, 4, 7, 31, 33, 64, 128, 255, 256, 260, 512, 515, 1000, 1024, 1028, 2048, 2056, 4096, 4100, 5003, 8192, 16384, 16388, 20001]


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_forward(dim, types):
    for rows, shift, w_type in ((1, 0, F32), (3, 0, BF16), (37, 1, F32), (8, 4, BF16)):
        x = made((rows, dim), types[0], shift, 1.0, 0.3, seed=dim + rows)
        w, b = made((dim,), w_type, shift, 0.3, 1.0, seed=1), made((dim,), w_type, shift, 0.5, seed=2)
        y, stats = Buffer(rows * dim, types[1], shift), Buffer(rows * 2, F32, shift)
        run(x, rows, dim, w, b, y, stats)
        check(x, rows, dim, w, b, y, stats)


def test_forward_without_weights_or_stats():
    for dim in (64, 515, 4096, 17000):
        x, y = made((5, dim), F32, 0, 2.0, -1.0), Buffer(5 * dim, F32, 0)
        w, b = made((dim,), F32, 0, 0.3, 1.0), made((dim,), F32, 0, 0.5)
        for ww, bb in ((None, None), (w, None), (None, b)):
            run(x, 5, dim, ww, bb, y, None)
            check(x, 5, dim, ww, bb, y, None)


MANY = [(70_000, 64, (BF16, BF16)), (20_011, 515, (BF16, BF16)), (5_000, 1024, (BF16, BF16)), (3_000, 4096, (BF16, BF16)), (700, 9000, (BF16, BF16)),
        (9_000, 256, (F32, F32)), (3_000, 1028, (F32, BF16)), (3_000, 1024, (BF16, F32)), (900, 2056, (F32, F32)), (90_000, 33, (F32, F32)),
        (200_000, 16, (BF16, BF16)), (3_000, 1001, (BF16, F32)), (1_500, 3333, (F32, F32)), (500, 6001, (F32, F32)), (300, 7000, (BF16, BF16)),
        (400, 8192, (F32, F32)), (200, 15_001, (F32, BF16)), (150, 16_384, (F32, F32)), (2_500, 768, (BF16, BF16))]


@pytest.mark.parametrize("rows,dim,types", MANY, ids=str)
def test_forward_of_many_rows(rows, dim, types):
    x = made((rows, dim), types[0], 0, 1.0, 0.3)
    w, b = made((dim,), F32, 0, 0.3, 1.0, seed=1), made((dim,), F32, 0, 0.5, seed=2)
    y, stats = Buffer(rows * dim, types[1], 0), Buffer(rows * 2, F32, 0)
    run(x, rows, dim, w, b, y, stats)
    check(x, rows, dim, w, b, y, stats)


# enough elements for several turns, where the elements to a thread follow from how rows of that length fill the device
TURNS = [(16_000, 264, (BF16, BF16)), (5_500, 768, (BF16, F32)), (2_000, 2304, (F32, BF16)), (1_000, 4104, (F32, F32)), (60_000, 72, (F32, F32)),
         (24_000, 515, (F32, F32)), (8_000, 643, (BF16, F32)), (500, 8200, (BF16, BF16)), (400, 12_288, (F32, F32)), (12_000, 385, (BF16, BF16)),
         (700, 12_296, (F32, F32)), (600, 14_000, (F32, BF16)), (500, 16_384, (BF16, F32)), (300, 12_296, (BF16, BF16)), (75, 10_001, (F32, F32)),
         (800, 12_287, (BF16, BF16)), (600, 9001, (F32, BF16)), (90, 16_400, (F32, BF16)), (200, 24_577, (BF16, F32)), (60, 49_152, (F32, F32)),
         (70, 49_153, (BF16, BF16)), (1, 65_536, (F32, F32)), (77, 65_544, (BF16, BF16)), (0, 9_001, (F32, F32)), (2_000, 2050, (F32, BF16)),
         (2_000, 2056, (F32, F32)), (8_000, 2001, (BF16, BF16))]


@pytest.mark.parametrize("rows,dim,types", TURNS, ids=str)
def test_forward_of_several_turns(rows, dim, types):
    test_forward_of_many_rows(rows, dim, types)


def test_rows_far_from_zero_and_constant_rows():
    """A mean 1000 times the deviation costs what the mean's own rounding costs, and no more; a constant row has no deviation."""
    for dim in (64, 1024, 4099, 17000):
        x = made((4, dim), F32, 0, 1.0, 1000.0)
        x.shaped[2] = 3.25
        x.shaped[3] = 0.0
        y, stats = Buffer(4 * dim, F32, 0), Buffer(8, F32, 0)
        run(x, 4, dim, None, None, y, stats)
        check(x, 4, dim, None, None, y, stats)
        assert (y.cpu().view(4, dim)[2:] == 0).all()


def test_no_rows_and_no_elements():
    y = Buffer(64, F32, 0)
    before = y.cpu()
    e = torch.empty(0, device="cuda")
    mqg.mqg_layer_norm(e, 0, 64, None, None, EPS, y.view)
    mqg.mqg_layer_norm(e, 7, 0, None, None, EPS, y.view)
    assert torch.equal(before.view(torch.int32), y.cpu().view(torch.int32))
    for dim in (64, 515, 1024, 4096, 6000, 17000):
        dw = torch.full((dim,), 3.0, device="cuda")
        db = torch.full((dim,), 4.0, device="cuda")
        work = torch.empty(mqg.mqg_layer_norm_workspace_floats(0, dim), device="cuda")
        mqg.mqg_layer_norm_grad(e, e, 0, dim, None, e, None, dw, db, work, add_into_grads=True)
        assert (dw == 3).all() and (db == 4).all()
        mqg.mqg_layer_norm_grad(e, e, 0, dim, None, e, None, dw, db, work)
        assert not dw.any() and not db.any()


def grad(dy, x, rows, dim, w, stats, dx, dw, db, add=False):
    work = Buffer(mqg.mqg_layer_norm_workspace_floats(rows, dim), F32, 0)
    mqg.mqg_layer_norm_grad(dy.view, x.view, rows, dim, None if w is None else w.view, stats.view, None if dx is None else dx.view,
                            None if dw is None else dw.view, None if db is None else db.view, work.view, add_into_grads=add)
    work.check()


def grad_plain(dy, x, w, stats):
    mu, r = stats[:, :1], stats[:, 1:]
    h, a = (x - mu) * r, w * dy
    m1, m2 = a.mean(-1, keepdim=True), (a * h).mean(-1, keepdim=True)
    off = r * U * (5 * a.abs() + (CHAIN + 4) * a.abs().mean(-1, keepdim=True) + (CHAIN + 10) * h.abs() * (a * h).abs().mean(-1, keepdim=True))
    return r * (a - m1 - h * m2), off, (dy * h).sum(0), dy.sum(0), (dy * h).abs().sum(0), dy.abs().sum(0)


def grad_check(dy, x, rows, dim, w, stats, dx, dw, db, before=None):
    one = torch.ones(dim, dtype=torch.float64)
    want, off, want_w, want_b, sum_w, sum_b = grad_plain(dy.cpu().view(rows, dim).double(), x.cpu().view(rows, dim).double(),
                                                         one if w is None else w.cpu().double(), stats.cpu().view(rows, 2).double())
    if dx is not None:
        got = dx.cpu().view(rows, dim)
        assert ((got.double() - want).abs() <= off * (1 + HALF[got.dtype]) + HALF[got.dtype] * want.abs() + 1e-40).all()
    for d, sums, total, own, k in ((dw, want_w, sum_w, 3, 0), (db, want_b, sum_b, 0, 1)):
        if d is None:
            continue
        total_off = (rows + own) * U * total                        # at most one addition in fp32 for every row
        if before is not None:
            sums = sums + before[k].double()
        got = d.cpu()
        assert ((got.double() - sums).abs() <= total_off * (1 + HALF[got.dtype]) + HALF[got.dtype] * sums.abs() + 1e-40).all()


def grad_case(rows, dim, types, shift=0, w_type=F32, dw_type=F32, seed=0):
    x = made((rows, dim), types[0], shift, 1.0, 0.3, seed)
    dy = made((rows, dim), types[1], shift, 1e-2, 1e-3, seed + 1)
    w = made((dim,), w_type, shift, 0.3, 1.0, seed + 2)
    _, mu, r, *_ = plain(x.cpu().view(rows, dim).double(), torch.ones(dim), torch.zeros(dim))
    stats = Buffer(rows * 2, F32, shift, torch.cat([mu, r], 1).float().view(-1))
    return dy, x, rows, dim, w, stats, Buffer(rows * dim, types[0], shift), Buffer(dim, dw_type, shift), Buffer(dim, dw_type, shift)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_gradient(dim, types):
    for rows, shift, w_type, dw_type in ((1, 0, F32, F32), (3, 0, BF16, BF16), (37, 1, F32, F32), (200, 4, BF16, F32)):
        c = grad_case(rows, dim, types, shift, w_type, dw_type, seed=dim + rows)
        grad(*c)
        grad_check(*c)


@pytest.mark.parametrize("rows,dim,types", MANY, ids=str)
def test_gradient_of_many_rows(rows, dim, types):
    c = grad_case(rows, dim, types)
    grad(*c)
    grad_check(*c)


@pytest.mark.parametrize("rows,dim,types", TURNS, ids=str)
def test_gradient_of_several_turns(rows, dim, types):
    test_gradient_of_many_rows(rows, dim, types)


def test_gradient_added_to_what_is_there():
    for dim in (64, 515, 4096, 17000):
        for dw_type in (F32, BF16):
            c = grad_case(50, dim, (F32, F32), dw_type=dw_type)
            for d in c[7:]:
                d.view.copy_(torch.randn(dim))
            before = [c[7].cpu(), c[8].cpu()]
            grad(*c, add=True)
            grad_check(*c, before=before)


def test_any_of_the_gradients_may_be_left_out():
    for dim in (64, 515, 4096, 17000):
        full = grad_case(50, dim, (F32, F32))
        grad(*full)
        for keep in range(1, 8):
            c = grad_case(50, dim, (F32, F32))
            out = [d if keep >> i & 1 else None for i, d in enumerate(c[6:])]
            grad(*c[:6], *out)
            for d, whole in zip(out, full[6:]):
                if d is not None:
                    assert torch.equal(d.cpu(), whole.cpu())
        c = grad_case(50, dim, (F32, F32))
        grad(*c[:4], None, *c[5:])
        grad_check(*c[:4], None, *c[5:])
        if dim < 17000:
            mqg.mqg_layer_norm_grad(c[0].view, c[1].view, 50, dim, None, c[5].view, c[6].view, None, None, None)


@pytest.mark.parametrize("rows,dim,types", [(50, 9001, (F32, F32)), (600, 14_000, (F32, F32)), (700, 12_288, (F32, BF16)), (50, 16_384, (BF16, BF16))], ids=str)
def test_any_of_the_gradients_of_long_rows_may_be_left_out(rows, dim, types):
    full = grad_case(rows, dim, types)
    grad(*full)
    for keep in (1, 2, 3, 4, 6):
        c = grad_case(rows, dim, types)
        out = [d if keep >> i & 1 else None for i, d in enumerate(c[6:])]
        grad(*c[:6], *out)
        for d, whole in zip(out, full[6:]):
            if d is not None:
                assert torch.equal(d.cpu(), whole.cpu())


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 129, 1000, 4097])
@pytest.mark.parametrize("dim", [1, 3, 64, 100, 515, 1024, 2050, 4096, 16400])
def test_every_row_is_counted_once(rows, dim):
    """Whole numbers with mu = 0 and r = 1: every sum is exact in fp32 in any order (below 2^24)."""
    if rows * dim > 20_000_000:
        pytest.skip("long")
    gen = torch.Generator().manual_seed(rows * 7 + dim)
    x = torch.randint(-8, 9, (rows, dim), generator=gen).float()
    dy = torch.randint(-8, 9, (rows, dim), generator=gen).float()
    for kind in (F32, BF16):
        stats = torch.tensor([0.0, 1.0]).repeat(rows, 1).cuda()
        bx, bdy = Buffer(rows * dim, kind, 0, x.view(-1).to(kind)), Buffer(rows * dim, kind, 0, dy.view(-1).to(kind))
        bs, dx, dw, db = Buffer(rows * 2, F32, 0, stats.view(-1)), Buffer(rows * dim, kind, 0), Buffer(dim, F32, 0), Buffer(dim, F32, 0)
        grad(bdy, bx, rows, dim, None, bs, dx, dw, db)
        assert torch.equal(dw.cpu(), (x * dy).sum(0)) and torch.equal(db.cpu(), dy.sum(0))
        dx.check()


def test_gradient_against_differences():
    """The directional derivative of sum(y c) with y as the forward pass computes it, from fp32 outputs read in 64 bits."""
    rows, dim = 6, 200
    x, w, b = made((rows, dim), F32, 0, 1.0, 0.2, 1), made((dim,), F32, 0, 0.3, 1.0, 2), made((dim,), F32, 0, 0.3, 0.0, 3)
    c = made((rows, dim), F32, 0, 1.0, 0.0, 4)
    y, stats = Buffer(rows * dim, F32, 0), Buffer(rows * 2, F32, 0)
    run(x, rows, dim, w, b, y, stats)
    dx, dw, db = Buffer(rows * dim, F32, 0), Buffer(dim, F32, 0), Buffer(dim, F32, 0)
    grad(c, x, rows, dim, w, stats, dx, dw, db)
    for target, d in ((x, dx), (w, dw), (b, db)):
        kept = target.cpu().clone()
        direction = torch.randn(kept.shape, generator=torch.Generator().manual_seed(5))
        values = []
        step = 2.0 ** -7
        for sign in (1, -1):
            target.view.copy_(kept + sign * step * direction)
            run(x, rows, dim, w, b, y, None)
            values.append((y.cpu().double() * c.cpu().double()).sum())
        target.view.copy_(kept)
        numeric = (values[0] - values[1]) / (2 * step)
        exact = (d.cpu().double() * direction.double()).sum()
        # error of the difference: step^2 / 6 of the third derivative (that of y along the direction is of the order of the
        # direction's own cube, a few of |c|), and the roundings of 1200 values of some 2^-22 each over 2 step
        assert abs(numeric - exact) <= 1e-3 * (c.cpu().norm() * direction.norm()).item(), (numeric, exact)


def test_captured_and_replayed():
    c = grad_case(300, 515, (BF16, BF16))
    y, stats = Buffer(300 * 515, BF16, 0), Buffer(600, F32, 0)
    work = torch.empty(mqg.mqg_layer_norm_workspace_floats(300, 515), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mqg.mqg_layer_norm(c[1].view, 300, 515, c[4].view, None, EPS, y.view, stats.view)
        mqg.mqg_layer_norm_grad(c[0].view, c[1].view, 300, 515, c[4].view, stats.view, c[6].view, c[7].view, c[8].view, work)
    for k in range(3):
        c[1].view.copy_(torch.randn(300 * 515))
        graph.replay()
        check(c[1], 300, 515, c[4], None, y, stats)
        grad_check(c[0], c[1], 300, 515, c[4], stats, *c[6:])


@pytest.mark.parametrize("rows,dim", [(90, 9001), (700, 12_288), (40, 16_400)])
def test_long_rows_captured_and_replayed_on_two_streams(rows, dim):
    cases = [grad_case(rows, dim, (F32, F32), seed=k) for k in range(2)]
    alone, graphs, streams = [], [], [torch.cuda.Stream() for _ in cases]
    for c, s in zip(cases, streams):
        grad(*c)
        alone.append([d.cpu() for d in c[6:]])
        work = torch.empty(mqg.mqg_layer_norm_workspace_floats(rows, dim), device="cuda")
        graphs.append((torch.cuda.CUDAGraph(), work))
        with torch.cuda.graph(graphs[-1][0], stream=s):
            mqg.mqg_layer_norm_grad(c[0].view, c[1].view, rows, dim, c[4].view, c[5].view, c[6].view, c[7].view, c[8].view, work)
        for d in c[6:]:
            d.view.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for (graph, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for c, want in zip(cases, alone):
        assert all(torch.equal(d.cpu(), w) for d, w in zip(c[6:], want))


def test_on_two_streams_at_once_behind_what_they_still_write():
    cases = [grad_case(2000, dim, (F32, F32)) for dim in (64, 1024)]
    alone = []
    for c in cases:
        grad(*c)
        alone.append([d.cpu() for d in c[6:]])
        for d in c[6:]:
            d.view.zero_()
        c[0].view.mul_(0.5)
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            torch.cuda._sleep(10_000_000)
            c[0].view.mul_(2.0)
            grad_work = torch.empty(mqg.mqg_layer_norm_workspace_floats(c[2], c[3]), device="cuda")
            mqg.mqg_layer_norm_grad(c[0].view, c[1].view, c[2], c[3], c[4].view, c[5].view, c[6].view, c[7].view, c[8].view, grad_work)
    torch.cuda.synchronize()
    for c, want in zip(cases, alone):
        assert all(torch.equal(d.cpu(), w) for d, w in zip(c[6:], want))


@pytest.mark.parametrize("dim", [1024, 515, 9001, 17000])
def test_offsets_beyond_32_bits(dim):
    rows = (1 << 32) // dim + 70
    n = rows * dim
    if torch.cuda.mem_get_info()[0] < 9 * n:
        pytest.skip("not enough device memory")
    x, dy = (torch.zeros(n, dtype=BF16, device="cuda") for _ in range(2))
    out = torch.empty(n, dtype=BF16, device="cuda")
    stats = torch.empty(2 * rows, device="cuda")
    spots = [0, rows // 2, rows - 5]
    c = grad_case(5, dim, (BF16, BF16))
    for at in spots:
        x[at * dim:(at + 5) * dim].copy_(c[1].view)
        dy[at * dim:(at + 5) * dim].copy_(c[0].view)
    y, s = Buffer(5 * dim, BF16, 0), Buffer(10, F32, 0)
    mqg.mqg_layer_norm(x, rows, dim, c[4].view, None, EPS, out, stats)
    run(c[1], 5, dim, c[4], None, y, s)
    check(c[1], 5, dim, c[4], None, y, s)
    for at in spots:
        assert torch.allclose(out[at * dim:(at + 5) * dim].cpu().float(), y.cpu().float(), rtol=2.0 ** -7, atol=1e-6)
        assert torch.allclose(stats[2 * at:2 * at + 10].cpu(), s.cpu(), rtol=1e-5, atol=1e-6)
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    work = torch.empty(mqg.mqg_layer_norm_workspace_floats(rows, dim), device="cuda")
    mqg.mqg_layer_norm_grad(dy, x, rows, dim, c[4].view, stats, out, dw, db, work)
    grad(c[0], c[1], 5, dim, c[4], s, *c[6:])
    for at in spots:
        got, want = out[at * dim:(at + 5) * dim].cpu().float(), c[6].cpu().float()
        assert torch.allclose(got, want, rtol=2.0 ** -6, atol=1e-6)
    # the other rows are zeros: three times the small sums, with roundings of every part
    for d, small in ((dw, c[7]), (db, c[8])):
        assert torch.allclose(d.cpu(), 3 * small.cpu(), rtol=1e-4, atol=1e-5)
