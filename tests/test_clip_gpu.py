"""The global norm of many gradient tensors, clipping in place, into a flat vector and in the server's update.

What the tolerance of the norm counts: a thread sums at most 33 squares in fp32, each at most 13 roundings deep (one of the
product, at most 7 of a chain, 5 joining the chains and the edge element), from there on in 64 bits.  All terms are positive,
so the sum of squares is off by at most 13 * 2^-24 of itself, its root by half of that, and rounding to fp32 adds 2^-24: 7.5 *
2^-24 in all, and 8 * 2^-24 with the second-order terms.  The factor has the same error.  Everything after the factor is
compared bit for bit with one rounding of the product."""
import math
import weakref

import pytest
import torch

import paper_1804_08066_b200 as mqg
from tests.buffers import Buffer, same_bits

pytestmark = pytest.mark.gpu
NORM_TOL = 8 * 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16

SIZES = {
    "none": [],
    "empty": [0, 0],
    "one": [1],
    "few": [0, 1, 5, 0, 33, 0],
    "tile": [4096],
    "edges": [4095, 4097, 8191, 8193, 1],
    "loop": [864, 32, 18_432, 64, 73_728, 128, 524_288, 256, 2_560, 10],
    "seventy": [(37 * i) % 501 for i in range(70)],
    "two_tables": [1 + (53 * i) % 97 for i in range(1500)],
    "long": [6_000_011, 7, 3_000_000],
    "nine_tiles": [8 * 4096 + 1],
    "32_tiles": [31 * 4096, 4095],
    "33_tiles": [31 * 4096 + 1, 4096],
    "32_wide_tiles": [31 * 8192, 8191],
    "32_tensors": [100 + i for i in range(32)],
    "33_tensors": [100 + i for i in range(33)],
}


def _types(kind, count):
    return [{"f32": F32, "bf16": BF16, "mixed": (F32, BF16)[i % 2]}[kind] for i in range(count)]


def _tensors(sizes, kind, shift=0, sigma=1e-3, seed=0):
    gen = torch.Generator().manual_seed(seed)
    values = [(torch.randn(s, generator=gen) * sigma * (1 + j % 5)).to(t) for j, (s, t) in enumerate(zip(sizes, _types(kind, len(sizes))))]
    return values, [Buffer(v.numel(), v.dtype, shift, v) for v in values]


def _norm64(values):
    return math.sqrt(math.fsum(float(v.double().square().sum()) for v in values))


def _scratch(count):
    floats = mqg.mqg_norm_workspace_floats(count)
    return Buffer(2, F32), Buffer(floats, F32, values=torch.full((floats,), float("nan")))


def _check_result(result, values, max_norm):
    norm, c = result.cpu().tolist()
    want, max_norm = _norm64(values), float(torch.tensor(max_norm, dtype=F32))     # the limit is passed in fp32
    if want > torch.finfo(F32).max * (1 + NORM_TOL):
        assert norm == math.inf                                                      # as fp32 holds it
    else:
        assert abs(norm - want) <= NORM_TOL * want
    if want <= max_norm * (1 - NORM_TOL):
        assert c == 1.0
    elif want > max_norm * (1 + NORM_TOL):
        assert abs(c - max_norm / want) <= NORM_TOL * c
    return torch.tensor(c, dtype=F32)


def _product(c, v, out):
    """One rounding to fp32, and one to the output's type."""
    return (c * v.float()).to(out)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES)
def test_norm_and_factor(sizes, kind, shift):
    values, bufs = _tensors(SIZES[sizes], kind, shift)
    want = _norm64(values)
    for max_norm in (0.0, 0.3 * want, 2.0 * want, math.inf):
        result, work = _scratch(len(bufs))
        mqg.mqg_grad_norm([b.view for b in bufs], max_norm, result.view, work.view)
        _check_result(result, values, max_norm)
        work.check()
    for b, v in zip(bufs, values):
        assert same_bits(b.cpu(), v)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES)
def test_clip_in_place(sizes, kind, shift):
    for ratio in (0.3, 2.0):
        values, bufs = _tensors(SIZES[sizes], kind, shift)
        max_norm = ratio * _norm64(values)
        result, work = _scratch(len(bufs))
        mqg.mqg_clip_grad_norm([b.view for b in bufs], max_norm, result.view, work.view)
        c = _check_result(result, values, max_norm)
        for b, v in zip(bufs, values):
            assert same_bits(b.cpu(), _product(c, v, v.dtype))


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES)
def test_flatten(sizes, kind, shift, out):
    values, bufs = _tensors(SIZES[sizes], kind, shift)
    total = sum(SIZES[sizes])
    for max_norm in (0.3 * _norm64(values), math.inf):
        flat = Buffer(total, out, (2 * shift) % 5)
        result, work = _scratch(len(bufs))
        mqg.mqg_clip_flatten([b.view for b in bufs], max_norm, flat.view, result.view, work.view)
        c = _check_result(result, values, max_norm)
        want = torch.cat([_product(c, v, out) for v in values]) if values else torch.empty(0, dtype=out)
        assert same_bits(flat.cpu(), want)
        for b, v in zip(bufs, values):
            assert same_bits(b.cpu(), v)


@pytest.mark.parametrize("kind", ["f32", "mixed"])
@pytest.mark.parametrize("factor", [1.0, 0.0, -0.37, 3.0])
def test_scale_by_a_given_factor(factor, kind):
    values, bufs = _tensors(SIZES["edges"] + SIZES["seventy"], kind, 1)
    f = torch.tensor([factor], device="cuda")
    mqg.mqg_scale_grads([b.view for b in bufs], f)
    for b, v in zip(bufs, values):
        assert same_bits(b.cpu(), _product(torch.tensor(factor), v, v.dtype))


@pytest.mark.parametrize("n", [1, 3, 4, 1023, 100_013, 3_000_001])
def test_apply_clipped_is_scale_then_apply(n):
    gen = torch.Generator().manual_seed(n)
    p, g = torch.randn(n, generator=gen), torch.randn(n, generator=gen) * 1e-2
    params, acc, factor, lr = Buffer(n, F32, values=p), Buffer(n, F32, values=g), torch.tensor([0.3], device="cuda"), 0.07
    mqg.mqg_apply_clipped(params.view, acc.view, lr, factor, n)
    assert same_bits(acc.cpu(), g)
    ref, scaled = p.cuda(), g.cuda()
    mqg.mqg_scale_grads([scaled], factor)
    mqg.mqg_apply(ref, scaled, lr, n)
    assert same_bits(params.cpu(), ref.cpu())
    # and the formula: roundings of the product (2^-24 of it) and of the sum (2^-24 of the result)
    step = float(torch.tensor(lr)) * float(factor.cpu()) * g.double()
    want = p.double() - step
    assert ((params.cpu().double() - want).abs() <= 1.01 * 2.0 ** -24 * (step.abs() + want.abs())).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("sigma", [1e-30, 1e-22, 1e18, 1e30, 1e37])
def test_squares_outside_fp32(sigma, kind):
    values, bufs = _tensors([5000, 3, 20_000], kind, 1, sigma)
    result, work = _scratch(3)
    max_norm = 0.5 * _norm64(values)
    mqg.mqg_grad_norm([b.view for b in bufs], max_norm, result.view, work.view)
    _check_result(result, values, max_norm)


def test_a_norm_that_fp32_does_not_hold_clips_all_the_same():
    values, bufs = _tensors([5000, 3, 20_000], "f32", 1, 1e37)
    result, work = _scratch(3)
    mqg.mqg_clip_grad_norm([b.view for b in bufs], 1e38, result.view, work.view)
    c = _check_result(result, values, 1e38)
    assert 0 < c < 1
    for b, v in zip(bufs, values):
        assert same_bits(b.cpu(), _product(c, v, F32))


def test_large_and_small_tensors_together():
    values = [torch.full((9000,), 2.0 ** -70), torch.full((3,), 2.0 ** 70), torch.zeros(70_000)]
    result, work = _scratch(3)
    mqg.mqg_grad_norm([v.cuda() for v in values], math.inf, result.view, work.view)
    _check_result(result, values, math.inf)
    mqg.mqg_grad_norm([v.cuda() for v in values[::2]], math.inf, result.view, work.view)
    _check_result(result, values[::2], math.inf)


def test_zeros_have_norm_zero_and_factor_one():
    result, work = _scratch(1)
    mqg.mqg_grad_norm([torch.zeros(10_000, device="cuda")], 0.0, result.view, work.view)
    assert result.cpu().tolist() == [0.0, 1.0]


@pytest.mark.parametrize("count", [0, 1, 32, 33, 1024, 1025, 1500])
def test_any_number_of_empty_tensors_have_norm_zero_and_factor_one(count):
    grads = [torch.empty(0, device="cuda", dtype=t) for t in _types("mixed", count)]
    for max_norm in (0.0, 0.5, math.inf):
        for call in (mqg.mqg_grad_norm, mqg.mqg_clip_grad_norm):
            result, work = _scratch(count)
            result.view.fill_(math.nan)
            call(grads, max_norm, result.view, work.view)
            assert result.cpu().tolist() == [0.0, 1.0]
            work.check()
        result, work, flat = *_scratch(count), Buffer(8, F32)
        result.view.fill_(math.nan)
        mqg.mqg_clip_flatten(grads, max_norm, flat.view, result.view, work.view)
        assert result.cpu().tolist() == [0.0, 1.0]
        assert (flat.cpu().view(torch.uint8) == 0x5A).all()
        work.check()


def test_what_is_not_finite():
    for at in (0, 4999, 9999):
        x = torch.ones(10_000)
        x[at] = math.inf
        result, work = _scratch(1)
        g = x.cuda()
        mqg.mqg_clip_grad_norm([g], 1.0, result.view, work.view)
        assert result.cpu().tolist() == [math.inf, 0.0]
        y = g.cpu()
        assert math.isnan(y[at]) and (torch.cat([y[:at], y[at + 1:]]) == 0).all()
        mqg.mqg_grad_norm([x.cuda()], math.inf, result.view, work.view)
        assert result.cpu().tolist() == [math.inf, 1.0]
        x[at] = math.nan
        g = x.cuda()
        mqg.mqg_clip_grad_norm([g], 1.0, result.view, work.view)
        assert all(math.isnan(r) for r in result.cpu().tolist()) and g.cpu().isnan().all()


def test_two_calls_agree_bit_for_bit_whatever_is_in_the_workspace():
    values, bufs = _tensors(SIZES["long"], "mixed", 1)
    got = []
    for fill in (0.0, float("nan"), 3.0):
        result, work = _scratch(3)
        work.view.fill_(fill)
        mqg.mqg_grad_norm([b.view for b in bufs], 1.0, result.view, work.view)
        got.append(result.cpu())
    assert same_bits(got[0], got[1]) and same_bits(got[0], got[2])


def test_scaling_the_scales_clips_an_encoded_gradient():
    """Clipping on the wire: the codes of a clipped gradient are those of the gradient, its scales the clipped ones."""
    n, bits, bucket = 70_000, 4, 512
    g = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() * 1e-2
    result, work = _scratch(1)
    codes = torch.zeros(mqg.mqg_code_words(n, bits), dtype=torch.int32, device="cuda")
    scales = torch.zeros(mqg.mqg_num_buckets(n, bucket), device="cuda")
    mqg.mqg_quantize(g, n, bits, bucket, 7, codes, scales)
    whole, clipped = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    mqg.mqg_dequant_accumulate([codes], [scales], 1, bits, n, whole, bucket)
    mqg.mqg_grad_norm([g], 0.5, result.view, work.view)
    mqg.mqg_scale_grads([scales], result.view[1:])
    mqg.mqg_dequant_accumulate([codes], [scales], 1, bits, n, clipped, bucket)
    c = float(result.cpu()[1])
    assert 0 < c < 1
    # roundings: the scaled scale, its quotient, the product, against quotient and product: 2^-24 each
    assert ((clipped.double() - c * whole.double()).abs() <= 5.1 * 2.0 ** -24 * c * whole.double().abs()).all()


def test_captured_replayed_and_on_another_stream():
    values, bufs = _tensors(SIZES["edges"], "mixed")
    total = sum(SIZES["edges"])
    result, work = _scratch(len(bufs))
    flat = Buffer(total, F32)
    grads = [b.view for b in bufs]

    def iteration():
        mqg.mqg_clip_flatten(grads, 0.05, flat.view, result.view, work.view)
        mqg.mqg_clip_grad_norm(grads, 0.05, result.view, work.view)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        iteration()
    torch.cuda.synchronize()
    c = _check_result(Buffer(2, F32, values=result.view), values, 0.05)
    once = [_product(c, v, v.dtype) for v in values]
    assert same_bits(flat.cpu(), torch.cat([_product(c, v, F32) for v in values]))
    for b, v in zip(bufs, once):
        assert same_bits(b.cpu(), v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iteration()
    for b, v in zip(bufs, values):
        b.view.copy_(v)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    # the second replay flattened what the first had clipped
    norm, again = result.cpu().tolist()
    assert abs(norm - 0.05) <= 0.05 * 2.0 ** -8
    flat.check()
    for b in bufs:
        b.check()


@pytest.mark.parametrize("size", [100, 200_000])
def test_tensors_that_an_iterable_makes_for_the_call_live_until_it_is_enqueued(size):
    """What is left of a temporary tensor when it is freed is overwritten at once, on the same stream: a call that is enqueued
    only afterwards would find zeros."""
    values = [torch.full((size,), float(j + 1)) for j in range(3)]

    def temporaries(kept):
        for v in values:
            kept.append(v.cuda())
            t = kept[-1].view(-1)
            weakref.finalize(t, kept[-1].zero_)
            yield t
            del t

    result, work = _scratch(3)
    for max_norm, call in ((math.inf, mqg.mqg_grad_norm), (0.5, mqg.mqg_grad_norm)):
        kept = []
        call(temporaries(kept), max_norm, result.view, work.view)
        _check_result(result, values, max_norm)
        assert all(int(k.count_nonzero()) == 0 for k in kept)          # freed by the end of the call
    kept, flat = [], Buffer(3 * size, F32)
    mqg.mqg_clip_flatten(temporaries(kept), 0.5, flat.view, result.view, work.view)
    c = _check_result(result, values, 0.5)
    assert same_bits(flat.cpu(), torch.cat([_product(c, v, F32) for v in values]))
    assert all(int(k.count_nonzero()) == 0 for k in kept)


def test_an_iterable_that_replaces_the_result_before_it_is_read():
    """Python code of the iterable runs before the other tensors' pointers are taken."""
    old, new, work = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda"), _scratch(1)[1]
    result = torch.zeros(2, device="cuda")
    result.set_(old)

    def items():
        result.set_(new)
        yield torch.full((4,), 1.5, device="cuda")

    mqg.mqg_grad_norm(items(), math.inf, result, work.view)
    assert result.tolist() == [3.0, 1.0] and new.tolist() == [3.0, 1.0] and old.tolist() == [0.0, 0.0]
