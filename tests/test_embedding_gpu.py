"""Rows of a table looked up for token ids, and the gradient of the table from sorted tokens.

The lookup has one rounding of the product (and one to bf16): compared bit for bit.  The gradient of a row with k tokens is a
sum in fp32: one after the other, or (some of those with 5 tokens and more, all with 64 and more) sums of at most 32 each, which are
added up in turn.  Each of them but two has 8 tokens at least, or 4 in a CTA of the one-launch form that has up to 256 tokens: no
term goes through more than 64 + k / 8 additions, or 8 + k / 4 with k up to 256, which is less, or k in
all where that is less, each off by at most 2^-24 of what it adds to, which is at most the sum of the magnitudes.  Then the product with the scale and, with add_into_grad, the sum with what was there (2^-24 each), and the
rounding to the output's type (half a step).  What these bounds cannot see in long runs, a token that is lost, taken twice or put
into another row, shows in sums of whole numbers, which are exact."""
import math
import pathlib
import subprocess
import sys
import threading

import pytest
import torch

import paper_1804_08066_b200 as mqg
from tests.buffers import Buffer, same_bits

pytestmark = pytest.mark.gpu
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64


def _ids(tokens, rows, kind, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        ids = torch.randint(0, max(1, rows), (tokens,), generator=gen)
    elif kind == "zipf":
        ids = (rows ** torch.rand(tokens, generator=gen, dtype=torch.float64)).long() - 1
    elif kind == "same":
        ids = torch.full((tokens,), rows - 1)
    elif kind == "empty":
        ids = torch.full((tokens,), -1)
    elif kind == "ascending":
        ids = torch.arange(tokens) * rows // max(1, tokens)
    else:                                    # outside the table on both sides
        ids = torch.randint(-rows - 1, 2 * rows + 1, (tokens,), generator=gen)
        ids[::7] = 2 ** 31 - 1 if dtype == I32 else 2 ** 32 + 1
        ids[3::7] = -2 ** 31 if dtype == I32 else -2 ** 63
    return ids.to(dtype)


def _held(ids, rows):
    return (ids.long() >= 0) & (ids.long() < rows)


def _lookup(table, ids, scale, out):
    held = _held(ids, table.shape[0])
    y = torch.zeros(ids.numel(), table.shape[1])
    y[held] = table[ids.long()[held]].float() * torch.tensor(scale, dtype=F32)
    return y.to(out)


SHAPES = [(1, 1, 1), (5, 7, 3), (3, 8, 1), (1000, 64, 500), (17, 257, 100), (300, 1024, 33), (9, 4100, 65), (50_021, 36, 4099)]


@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("shape", SHAPES)
def test_lookup(shape, shift, types):
    rows, dim, tokens = shape
    gen = torch.Generator().manual_seed(rows + dim)
    table = torch.randn(rows, dim, generator=gen).to(types[0])
    t = Buffer(rows * dim, types[0], shift, table.flatten())
    for kind, dtype in (("uniform", I64), ("zipf", I32), ("outside", I64), ("outside", I32)):
        ids = _ids(tokens, rows, kind, dtype)
        out = Buffer(tokens * dim, types[1], (3 * shift) % 5)
        mqg.mqg_embedding(t.view, rows, dim, Buffer(tokens, dtype, shift, ids).view, tokens, 1.7, out.view)
        assert same_bits(out.cpu(), _lookup(table, ids, 1.7, types[1]).flatten())
    t.check()


@pytest.mark.parametrize("dim", [4, 8, 12, 131_068, 131_072, 131_076, 400_000])
def test_lookup_of_rows_of_one_and_of_very_many_words(dim):
    rows, tokens = 3, 1500 if dim < 100 else 5
    table = torch.randn(rows, dim, generator=torch.Generator().manual_seed(dim))
    for kind in ("uniform", "outside"):
        ids, out = _ids(tokens, rows, kind, I64), Buffer(tokens * dim, F32)
        mqg.mqg_embedding(table.cuda(), rows, dim, ids.cuda(), tokens, -1.7, out.view)
        assert same_bits(out.cpu(), _lookup(table, ids, -1.7, F32).flatten())


def test_lookup_of_nothing_and_from_nothing():
    ids, out = torch.zeros(4, dtype=I64, device="cuda"), Buffer(12, F32)
    mqg.mqg_embedding(torch.empty(0, device="cuda"), 0, 3, ids, 4, 1.0, out.view)
    assert (out.cpu() == 0).all()
    out = Buffer(12, F32)
    before = out.raw.clone()
    mqg.mqg_embedding(torch.ones(15, device="cuda"), 5, 3, ids, 0, 1.0, out.view)
    mqg.mqg_embedding(torch.ones(15, device="cuda"), 5, 0, ids, 4, 1.0, out.view)
    assert (out.raw == before).all()


def test_rows_behind_the_last_token_stay():
    out = Buffer(100 * 8, BF16)
    mqg.mqg_embedding(torch.ones(40, device="cuda"), 5, 8, torch.zeros(64, dtype=I64, device="cuda"), 33, 1.0, out.view)
    got = out.cpu()
    assert (got[:33 * 8] == 1).all() and (got[33 * 8:].view(torch.int16) == 0x5A5A).all()


def _gradient(dout, ids, rows, scale, old):
    """The formula in 64 bits, and how far fp32 may be off it before the last rounding."""
    held = _held(ids, rows)
    at, d = ids.long()[held], dout.double()[held]
    total = torch.zeros(rows, dout.shape[1], dtype=torch.float64).index_add_(0, at, d) * scale
    size = torch.zeros(rows, dout.shape[1], dtype=torch.float64).index_add_(0, at, d.abs()) * abs(scale)
    k = torch.zeros(rows, dtype=torch.float64).index_add_(0, at, torch.ones(at.numel(), dtype=torch.float64))
    depth = torch.minimum(k, 64 + k / 8)
    off = (depth[:, None] * size + total.abs()) * 2.0 ** -24
    if old is not None:
        total = total + old.double()
        off = off + total.abs() * 2.0 ** -24
    return total, off * 1.001, k > 0


def _check_gradient(shape, kind, id_type, types, add, shift=0, scale=1.3, seed=0):
    rows, dim, tokens = shape
    gen = torch.Generator().manual_seed(seed + tokens)
    ids = _ids(tokens, rows, kind, id_type, seed)
    dout = torch.randn(tokens, dim, generator=gen).to(types[0])
    if tokens:
        dout[~_held(ids, rows)] = math.nan                            # empty places hold what they like
    old = torch.randn(rows, dim, generator=gen).to(types[1])
    scale = float(torch.tensor(scale, dtype=F32))
    want, off, used = _gradient(dout, ids, rows, scale, old if add else None)
    floats = mqg.mqg_embedding_workspace_floats(tokens, rows, dim)
    d = Buffer(tokens * dim, types[0], shift, dout.flatten())
    i = Buffer(tokens, id_type, shift, ids)
    got = []
    for fill in (float("nan"), 0.0):
        g = Buffer(rows * dim, types[1], (3 * shift) % 5, old.flatten())
        w = Buffer(floats, F32, values=torch.full((floats,), fill))
        mqg.mqg_embedding_grad(d.view, i.view, tokens, rows, dim, scale, g.view, w.view, add_into_grad=add)
        got.append(g.cpu().view(rows, dim))
        w.check()
    assert same_bits(got[0], got[1])                                  # reproducible, whatever the workspace held
    y = got[0].double()
    half_step = torch.finfo(types[1]).eps / 2 if types[1] == BF16 else 0.0   # fp32: counted in `off`
    assert ((y - want).abs() <= off + half_step * (want.abs() + off)).all()
    if add:
        assert same_bits(got[0][~used], old[~used])
    else:
        assert (got[0][~used] == 0).all()


GRAD_SHAPES = [(1, 1, 1), (5, 7, 3), (3, 8, 40), (1000, 64, 2048), (17, 257, 100), (300, 1024, 33), (9, 4100, 65),
               (40_000, 36, 4099), (70_001, 4, 20_000), (3, 130, 9000)]


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["uniform", "zipf", "outside"])
@pytest.mark.parametrize("shape", GRAD_SHAPES)
def test_gradient(shape, kind, add):
    _check_gradient(shape, kind, I64, (F32, F32), add)
    _check_gradient(shape, kind, I32, (BF16, F32), add, shift=1)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_gradient_of_each_type_and_alignment(types, shift, add):
    for shape in ((50, 24, 300), (50, 20, 300), (50, 18, 300), (50, 17, 300), (50, 520, 70)):
        _check_gradient(shape, "zipf", I64, types, add, shift)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("tokens", [0, 1, 31, 32, 33, 64, 65, 96, 1000, 8192, 8193, 30_000])
@pytest.mark.parametrize("kind", ["same", "empty", "ascending"])
def test_gradient_of_long_and_of_missing_runs(kind, tokens, add):
    _check_gradient((40, 12, tokens), kind, I64, (F32, F32), add)
    _check_gradient((40, 12, tokens), kind, I32, (BF16, BF16), add)


@pytest.mark.parametrize("rows", [1, 2, 255, 256, 257, 65_535, 65_536, 65_537, 1 << 20, (1 << 24) + 3])
def test_gradient_of_tables_at_the_digits_edges(rows):
    _check_gradient((rows, 2, 10_000), "uniform", I64, (F32, F32), False)
    _check_gradient((rows, 1, 300), "outside", I32, (F32, F32), True)


def _check_whole_numbers(shape, kind, id_type, types, add, shift=0, seed=0):
    """Sums of whole numbers that differ from token to token and from column to column: below 2^23 in halves, so that every
    partial sum, the product with 0.5 and the sum with what was there are exact, and a bf16 result is rounded once."""
    rows, dim, tokens = shape
    ids = _ids(tokens, rows, kind, id_type, seed)
    t, c = torch.arange(tokens)[:, None], torch.arange(dim)[None, :]
    dout = 1 + (7 * t + 5 * (t // 61) + 3 * c) % 61
    old = (11 * torch.arange(rows)[:, None] + c) % 201 - 100
    held = _held(ids, rows)
    total = torch.zeros(rows, dim, dtype=torch.int64).index_add_(0, ids.long()[held], dout[held])
    assert int(total.max()) < 2 ** 24 - 512
    want = (total.double() * 0.5 + (old if add else 0)).to(F32).to(types[1])
    grad = Buffer(rows * dim, types[1], (3 * shift) % 5, old.to(types[1]).flatten())
    floats = mqg.mqg_embedding_workspace_floats(tokens, rows, dim)
    work = Buffer(floats, F32, values=torch.full((floats,), math.nan))
    mqg.mqg_embedding_grad(Buffer(tokens * dim, types[0], shift, dout.to(types[0]).flatten()).view,
                           Buffer(tokens, id_type, shift, ids).view, tokens, rows, dim, 0.5, grad.view, work.view, add_into_grad=add)
    assert same_bits(grad.cpu().view(rows, dim), want)
    work.check()


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("dim", [17, 18, 20, 24])
@pytest.mark.parametrize("tokens", [5, 33, 250, 257, 2048, 8192, 8193, 16_385, 65_537, 131_073, 150_001])
def test_every_token_of_long_runs_counts_once(tokens, dim, types, add):
    for rows, kind in ((40, "same"), (300, "zipf")):
        _check_whole_numbers((rows, dim, tokens), kind, I64, types, add)
    _check_whole_numbers((300, dim, tokens), "zipf", I32, types, add, shift=1, seed=1)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("shape", [(40, 2055, 2048), (500, 801, 4097), (3, 1536, 2049), (20_000, 3146, 1000), (2000, 515, 10_007)])
def test_every_token_counts_once_in_wide_rows(shape, types, add):
    for kind in ("same", "zipf", "ascending"):
        _check_whole_numbers(shape, kind, I64, types, add)


@pytest.mark.parametrize("most_ctas", [8, 4, 2, 1])
@pytest.mark.parametrize("shape", [(300, 1600, 2049), (500, 800, 4097), (50_000, 3, 8193), (70_001, 5, 16_385), (40_000, 3, 65_537), (300, 7, 131_072),
                                   (9000, 4, 140_001)])
def test_gradient_where_the_device_holds_no_large_cluster(shape, most_ctas):
    """The order of the sums does not depend on how the tokens are sorted: the same bits."""
    rows, dim, tokens = shape
    dout = torch.randn(tokens, dim, generator=torch.Generator().manual_seed(4)).cuda()
    for kind, dtype in (("zipf", I64), ("outside", I32)):
        ids = _ids(tokens, rows, kind, dtype).cuda()
        floats = mqg.mqg_embedding_workspace_floats(tokens, rows, dim)
        got = []
        for most in (0, most_ctas):
            grad, work = Buffer(rows * dim, F32), Buffer(floats, F32, values=torch.full((floats,), math.nan))
            mqg.mqg_test_sort_cluster(most)
            try:
                mqg.mqg_embedding_grad(dout, ids, tokens, rows, dim, 0.7, grad.view, work.view)
            finally:
                mqg.mqg_test_sort_cluster(0)
            got.append(grad.cpu())
            work.check()
        assert same_bits(*got)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["zipf", "uniform", "outside"])
@pytest.mark.parametrize("tokens", [2047, 2049, 16_385, 65_537, 131_072, 131_073, 150_001])
def test_gradient_by_the_sort_of_each_size(tokens, kind, add):
    _check_gradient((50_000, 3, tokens), kind, I64, (F32, F32), add)
    _check_gradient((300, 4, tokens), kind, I32, (BF16, F32), add, shift=1)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("kind", ["same", "zipf", "uniform", "outside"])
@pytest.mark.parametrize("tokens", [1, 8, 9, 250, 1024, 1025, 2048, 4097, 8191])
def test_gradient_of_few_tokens(tokens, kind, add):
    for rows, dim in ((1, 9), (2, 33), (147, 32), (149, 31), (1000, 8), (9500, 40)):
        _check_gradient((rows, dim, tokens), kind, I32, (F32, BF16), add, shift=1)
        _check_gradient((rows, dim, tokens), kind, I64, (BF16, F32), add)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("shape", [(50, 384, 8192), (50, 385, 8192), (50, 24, 8193), (20, 4736, 600), (20, 4737, 600), (1 << 24, 1, 100), (131_072, 64, 40), (131_073, 64, 40), (64_527, 65, 40), (64_528, 65, 40),
                                   (2, 200_000, 7), (3, 250_000, 7)])
def test_gradient_where_one_launch_ends(shape, add):
    _check_gradient(shape, "zipf", I64, (F32, F32), add)
    _check_gradient(shape, "outside", I64, (F32, F32), add)


@pytest.mark.parametrize("shape", [(40_000, 1024, 33_000), (33_333, 1040, 33_000), (33_000, 4096, 8200), (260_000, 160, 262_144)])
def test_zeros_beside_rows_in_use_when_both_exceed_l2(shape):
    rows, dim, tokens = shape
    ids = _ids(tokens, rows, "outside" if rows == 40_000 else "zipf", I64)
    held = _held(ids, rows)
    d = torch.ones(tokens, dim, device="cuda")
    grad = torch.full((rows, dim), math.nan, device="cuda")
    w = torch.empty(mqg.mqg_embedding_workspace_floats(tokens, rows, dim), device="cuda")
    for _ in range(2):
        mqg.mqg_embedding_grad(d, ids.cuda(), tokens, rows, dim, 0.5, grad, w)
    count = torch.zeros(rows).index_add_(0, ids[held], torch.ones(int(held.sum())))       # whole numbers: sums are exact
    assert (grad.cpu() == 0.5 * count[:, None]).all()


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("shape", [(40_000, 1024, 33_000), (33_333, 1040, 33_000), (33_000, 4096, 8200), (260_000, 160, 140_000),
                                   (30_011, 515, 10_007), (3000, 8200, 9000), (900, 20_001, 9001), (70_000, 3, 9000), (1025, 7, 40_000)])
def test_rows_without_tokens_are_zero_whatever_the_call_before_left(shape, types):
    """Calls with other ids each time, with one workspace, into a gradient that holds NaN: nothing of the call before may show.
    Whole numbers: sums are exact, and a bf16 result is rounded once."""
    rows, dim, tokens = shape
    d = torch.ones(tokens, dim, device="cuda", dtype=types[0])
    grad = torch.empty(rows, dim, device="cuda", dtype=types[1])
    w = torch.empty(mqg.mqg_embedding_workspace_floats(tokens, rows, dim), device="cuda")
    for seed, kind in enumerate(("zipf", "outside", "same", "uniform", "zipf", "empty")):
        ids = _ids(tokens, rows, kind, I64, seed).cuda()
        grad.fill_(math.nan)
        mqg.mqg_embedding_grad(d, ids, tokens, rows, dim, 0.5, grad, w)
        held = (ids >= 0) & (ids < rows)
        count = torch.zeros(rows, device="cuda").index_add_(0, ids[held], torch.ones(tokens, device="cuda")[held])
        assert bool((grad == (0.5 * count[:, None]).to(types[1])).all()), kind


def test_gradient_by_differences():
    """<R, lookup(table)> is linear in the table: its central difference is the gradient of R."""
    rows, dim, tokens, scale, h = 6, 5, 40, 0.75, 0.5
    gen = torch.Generator().manual_seed(1)
    ids = _ids(tokens, rows, "zipf", I64).cuda()
    r = torch.randn(tokens, dim, generator=gen).cuda()
    table = torch.randn(rows, dim, generator=gen).cuda()
    grad = torch.zeros(rows, dim, device="cuda")
    w = torch.zeros(mqg.mqg_embedding_workspace_floats(tokens, rows, dim), device="cuda")
    mqg.mqg_embedding_grad(r, ids, tokens, rows, dim, scale, grad, w)

    def value(t):
        out = torch.zeros(tokens, dim, device="cuda")
        mqg.mqg_embedding(t, rows, dim, ids, tokens, scale, out)
        return float((out.double() * r.double()).sum())

    for v in range(rows):
        for c in range(dim):
            up, down = table.clone(), table.clone()
            up[v, c] += h
            down[v, c] -= h
            # at most 40 products, each off by 2^-24 of |table +- h| < 8 and |r| < 8, twice over 2 h
            assert abs((value(up) - value(down)) / (2 * h) - float(grad[v, c])) < 40 * 64 * 2.0 ** -23


@pytest.mark.parametrize("tokens", [3000, 20_000, 140_000])
def test_gradient_captured_replayed_and_on_another_stream(tokens):
    rows, dim = 500, 64
    ids = [_ids(tokens, rows, "zipf", I64, seed).cuda() for seed in (0, 1)]
    dout = torch.randn(tokens, dim, generator=torch.Generator().manual_seed(2)).cuda()
    floats = mqg.mqg_embedding_workspace_floats(tokens, rows, dim)
    want = []
    for i in ids:
        g = torch.empty(rows, dim, device="cuda")
        mqg.mqg_embedding_grad(dout, i, tokens, rows, dim, 2.0, g, torch.empty(floats, device="cuda"))
        want.append(g.cpu())
    side, held, g, out = torch.cuda.Stream(), ids[0].clone(), torch.empty(rows, dim, device="cuda"), torch.empty(tokens, dim, device="cuda")
    w = torch.empty(floats, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mqg.mqg_embedding_grad(dout, held, tokens, rows, dim, 2.0, g, w)
    torch.cuda.synchronize()
    assert same_bits(g.cpu(), want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mqg.mqg_embedding_grad(dout, held, tokens, rows, dim, 2.0, g, w)
        mqg.mqg_embedding(g, rows, dim, held, tokens, 1.0, out)
    for k in (1, 0, 1):
        held.copy_(ids[k])
        g.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(g.cpu(), want[k])
        assert same_bits(out.cpu(), _lookup(want[k], ids[k].cpu(), 1.0, F32))


@pytest.mark.parametrize("shape", [(50, 24, 700), (3000, 40, 12_000)])
def test_two_gradients_at_once_and_one_with_what_the_stream_still_writes(shape):
    """Calls on two streams with workspaces of their own, and a call whose ids and output gradient a launch just before it
    writes."""
    rows, dim, tokens = shape
    gen = torch.Generator().manual_seed(3)
    ids = _ids(tokens, rows, "zipf", I64).cuda()
    dout = torch.randn(tokens, dim, generator=gen).cuda()
    floats = mqg.mqg_embedding_workspace_floats(tokens, rows, dim)
    want = torch.empty(rows, dim, device="cuda")
    mqg.mqg_embedding_grad(dout, ids, tokens, rows, dim, 2.0, want, torch.empty(floats, device="cuda"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    held = [[torch.full_like(ids, -1), torch.zeros_like(dout), torch.full((rows, dim), math.nan, device="cuda"),
             torch.empty(floats, device="cuda")] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (i, d, g, w) in zip(streams, held):
            with torch.cuda.stream(s):
                i.copy_(ids)
                d.copy_(dout)
                g.fill_(math.nan)
                mqg.mqg_embedding_grad(d, i, tokens, rows, dim, 2.0, g, w)
                i.fill_(-1)
                d.zero_()
    torch.cuda.synchronize()
    for _, _, g, _ in held:
        assert same_bits(g.cpu(), want.cpu())


def test_no_tokens_set_the_gradient_to_zero_after_what_the_stream_still_writes():
    grad = torch.empty(4_000_001, device="cuda")
    ids, w = torch.empty(0, dtype=I64, device="cuda"), torch.empty(0, device="cuda")
    for _ in range(10):
        grad.fill_(math.nan)
        mqg.mqg_embedding_grad(grad, ids, 0, 4_000_001, 1, 1.0, grad, w)
    assert (grad.cpu() == 0).all()


def test_a_table_beyond_32_bit_offsets():
    rows, dim = 70_000, 1 << 16                      # 4.6 * 10^9 elements of bf16
    table = torch.zeros(rows, dim, dtype=BF16, device="cuda")
    ids = torch.tensor([rows - 1, 0, 65_536, rows, rows - 1, -1], device="cuda")
    table[rows - 1], table[65_536] = 3, 5
    out = torch.empty(6, dim, dtype=F32, device="cuda")
    mqg.mqg_embedding(table, rows, dim, ids, 6, 2.0, out)
    assert [float(x) for x in out[:, -1]] == [6, 0, 10, 0, 6, 0] and [float(x) for x in out[:, 0]] == [6, 0, 10, 0, 6, 0]
    w = torch.empty(mqg.mqg_embedding_workspace_floats(6, rows, dim), device="cuda")
    mqg.mqg_embedding_grad(out, ids, 6, rows, dim, 1.0, table, w, add_into_grad=True)
    assert [float(table[r, c]) for r in (rows - 1, 65_536, 0, 1) for c in (0, dim - 1)] == [15, 15, 15, 15, 0, 0, 0, 0]
    mqg.mqg_embedding_grad(out, ids, 6, rows, dim, 1.0, table, w)
    assert [float(table[r, c]) for r in (rows - 1, 65_536, 0, 1) for c in (0, dim - 1)] == [12, 12, 10, 10, 0, 0, 0, 0]


FIRST_CALLS = '''
import torch
import paper_1804_08066_b200 as mqg
rows = 500
for tokens, dim in ((1000, 64), (2000, 1600), (9000, 64), (20_000, 64), (140_000, 64)):
    ids, d = torch.arange(tokens, device="cuda") * 7 % rows, torch.ones(tokens, dim, device="cuda")
    g, out = torch.empty(rows, dim, device="cuda"), torch.empty(tokens, dim, device="cuda")
    w = torch.empty(mqg.mqg_embedding_workspace_floats(tokens, rows, dim), device="cuda")
    want = torch.bincount(ids, minlength=rows).float()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mqg.mqg_embedding_grad(d, ids, tokens, rows, dim, 1.0, g, w)
        mqg.mqg_embedding(g, rows, dim, ids, tokens, 1.0, out)
    for _ in range(2):
        g.fill_(float("nan"))
        graph.replay()
    assert bool((g == want[:, None]).all()) and bool((out == want[ids][:, None]).all()), tokens
'''


def test_the_first_calls_of_a_process_may_be_captured():
    subprocess.run([sys.executable, "-c", FIRST_CALLS], check=True, timeout=300, cwd=pathlib.Path(__file__).resolve().parent.parent)


def test_gradients_from_several_threads():
    """Streams and workspaces of their own; the calls run without the interpreter lock."""
    right = []

    def work(seed):
        with torch.cuda.stream(torch.cuda.Stream()):
            for tokens, dim in ((9000, 64), (20_000, 64), (140_000, 16), (2000, 1600), (500, 64)):
                rows = 500 + seed
                ids, d = torch.arange(tokens, device="cuda") * 7 % rows, torch.ones(tokens, dim, device="cuda")
                g = torch.empty(rows, dim, device="cuda")
                w = torch.empty(mqg.mqg_embedding_workspace_floats(tokens, rows, dim), device="cuda")
                for _ in range(20):
                    mqg.mqg_embedding_grad(d, ids, tokens, rows, dim, 1.0, g, w)
                right.append(bool((g == torch.bincount(ids, minlength=rows)[:, None]).all()))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert right == [True] * 20
