"""AdamW over many tensors against its formulas: m and v bit for bit with fp32 operations rounded one by one, parameters within
the roundings of the 64-bit result, codes and scales of states in 8 bits bit for bit."""
import math
import pathlib
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .adamw_plain import BLOCK, E4M3, E5M2, decode, moments32, step64, step8
from .buffers import Buffer

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: 0.0, BF16: 2.0 ** -8}                      # of the parameter's own rounding, relative


class Lists:
    """Tensors of the given sizes, each a guarded buffer `shift` elements off a boundary."""

    def __init__(self, sizes, p_type=F32, g_type=F32, eight=False, shift=0, seed=0, zeros=False):
        rng = np.random.default_rng(seed)
        self.sizes, self.eight = sizes, eight
        scale = [10.0 ** rng.uniform(-5, -1) for _ in sizes]

        def made(values, dtype):
            return [Buffer(v.size, dtype, shift, torch.from_numpy(v).cuda().to(dtype)) for v in values]

        def bits(values, dtype):
            out = [Buffer(v.size, torch.uint8, shift, torch.from_numpy(v).cuda()) for v in values]
            for b in out:
                b.view = b.view.view(dtype)
            return out

        self.p = made([rng.normal(0, 0.05, n).astype(np.float32) for n in sizes], p_type)
        self.g = made([(rng.normal(0, 1, n) * s).astype(np.float32) for n, s in zip(sizes, scale)], g_type)
        keep = 0.0 if zeros else 1.0
        if eight:
            blocks = [-(-n // BLOCK) for n in sizes]
            self.m = bits([(rng.integers(0, 0x7F, n) | rng.integers(0, 2, n) << 7).astype(np.uint8) * int(keep) for n in sizes],
                          torch.float8_e4m3fn)
            self.v = bits([rng.integers(0x30, 0x7C, n).astype(np.uint8) * int(keep) for n in sizes], torch.float8_e5m2)
            self.s = made([(rng.uniform(0.5, 1, (b, 2)) * [s / 448, s * s / 57344] * keep).astype(np.float32).reshape(-1)
                           for b, s in zip(blocks, scale)], F32)
        else:
            self.m = made([(rng.normal(0, 0.3, n) * s * keep).astype(np.float32) for n, s in zip(sizes, scale)], F32)
            self.v = made([(rng.uniform(0, 2, n) * s * s * keep).astype(np.float32) for n, s in zip(sizes, scale)], F32)
            self.s = []

    def tensors(self):
        lists = [[b.view for b in x] for x in (self.p, self.g, self.m, self.v)]
        return lists + [[b.view for b in self.s]] if self.eight else lists

    def step(self, t, decays=0.1, seed=7, **more):
        hyper = {**HYPER, "step": t, **more}
        if self.eight:
            mqg.mqg_adamw8(*self.tensors(), decays, seed=seed, **hyper)
        else:
            mqg.mqg_adamw(*self.tensors(), decays, **hyper)

    def state(self):
        """Everything on the host: values of p and g, m and v (codes if in 8 bits), scales."""
        raw = lambda b: b.cpu().view(torch.uint8).numpy().copy() if self.eight else b.cpu().numpy().copy()  # noqa: E731
        return {"p": [b.cpu().double().numpy() for b in self.p], "g": [b.cpu().float().numpy() for b in self.g],
                "m": [raw(b) for b in self.m], "v": [raw(b) for b in self.v],
                "s": [b.cpu().numpy().reshape(-1, 2).copy() for b in self.s]}


def same(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and a.tobytes() == b.tobytes()


def check(lists, before, after, t, decays, k=1.0, seed=7, **more):
    hyper = {**HYPER, **more}
    blocks = 0
    for j, n in enumerate(lists.sizes):
        decay = float(np.float32(decays if isinstance(decays, (int, float)) else decays[j]))
        p, g, m, v = (before[x][j] for x in "pgmv")
        if n == 0:
            continue
        if lists.eight:
            want, slack, m2, v2, s2 = step8(p, g, m, v, before["s"][j], blocks, seed=seed, step=t, k=k, decay=decay, **hyper)
            assert same(after["s"][j], s2)
            blocks += -(-n // BLOCK)
        else:
            want, _, _, slack = step64(p, g, m, v, step=t, k=k, decay=decay, **hyper)
            m2, v2 = moments32(g, m, v, beta1=hyper["beta1"], beta2=hyper["beta2"], k=k)
        assert same(after["m"][j], m2), (j, n)
        assert same(after["v"][j], v2), (j, n)
        off = np.abs(after["p"][j] - want)
        assert (off <= slack * (1 + ROUND[lists.p[j].view.dtype]) + ROUND[lists.p[j].view.dtype] * np.abs(want)).all(), (j, n, off.max())
        assert same(after["g"][j], g)


SIZES = [[1], [255, 256, 257], [0, 3, 0, 2049, 0], [64, 7, 1000, 513, 4096, 31, 1, 2048, 10]]


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)], ids=str)
def test_steps(types, shift, eight):
    for k, sizes in enumerate(SIZES):
        lists = Lists(sizes, *types, eight=eight, shift=shift, seed=k)
        decays = [0.1 * (j % 2) for j in range(len(sizes))]
        for t in (1, 2, 1000):
            before = lists.state()
            lists.step(t, decays)
            check(lists, before, lists.state(), t, decays)


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_the_first_step_from_zeros(eight):
    lists = Lists([300, 5], eight=eight, zeros=True)
    before = lists.state()
    lists.step(1, 0.0)
    after = lists.state()
    check(lists, before, after, 1, 0.0)
    for p, q, g in zip(before["p"], after["p"], before["g"]):        # the first step is lr * sign(g) wherever |g| is far above eps
        big = np.abs(g) > 1e-4
        assert np.allclose((p - q)[big], HYPER["lr"] * np.sign(g)[big], rtol=1e-3, atol=2.0 ** -24)


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("count", [17, 97, 449, 900])
def test_many_tensors_and_types_at_once(count, eight):
    """More tensors than a launch's table holds, of both types, slices of one vector in any order."""
    rng = np.random.default_rng(count)
    sizes = [int(n) for n in rng.integers(0, 60, count)]
    sizes[count // 2], sizes[-1] = 5000, 0
    lists = Lists(sizes, F32, F32, eight=eight, shift=1, seed=count)
    other = Lists(sizes, BF16, BF16, eight=eight, shift=3, seed=count + 1)
    for j in range(0, count, 3):
        lists.p[j], lists.g[(j + 1) % count] = other.p[j], other.g[(j + 1) % count]
    decays = rng.uniform(0, 0.5, count).tolist()
    before = lists.state()
    lists.step(3, decays)
    check(lists, before, lists.state(), 3, decays)


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_scale_and_factor(eight):
    for f in (0.25, 0.3, 1e-3):
        lists = Lists([1000, 33], eight=eight)
        before = lists.state()
        lists.step(5, grad_scale=1 / 3, factor=torch.tensor([f], device="cuda"))
        k = np.float32(1 / 3) * np.float32(f)
        check(lists, before, lists.state(), 5, 0.1, k=k)
    for f in (math.nan, math.inf, -math.inf, 0.0):
        lists = Lists([1000, 33], eight=eight)
        before = lists.state()
        lists.step(5, factor=torch.tensor([f], device="cuda"))
        after = lists.state()
        assert all(same(a, b) for x in before for a, b in zip(before[x], after[x]))


def test_a_gradient_with_a_nan_changes_nothing():
    """The norm's factor of such a gradient, as the trainer passes it on."""
    for bad in (math.nan, math.inf):
        lists = Lists([1000, 33])
        lists.g[1].view[7] = bad
        result, work = torch.empty(2, device="cuda"), torch.empty(mqg.mqg_norm_workspace_floats(2), device="cuda")
        before = lists.state()
        mqg.mqg_grad_norm([b.view for b in lists.g], 1.0, result, work)
        lists.step(5, factor=result[1:])
        after = lists.state()
        assert all(same(a, b) for x in "pmv" for a, b in zip(before[x], after[x]))


def corrections(t):
    return torch.tensor([HYPER["lr"], 1 - HYPER["beta1"] ** t, 1 - HYPER["beta2"] ** t, t], dtype=torch.float64).float()


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_replays_of_a_captured_step_are_the_steps(eight):
    eager, captured = Lists([1000, 33, 5000], eight=eight), Lists([1000, 33, 5000], eight=eight)
    schedule = corrections(1).cuda()
    before = captured.state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step(0, lr=0.5, schedule=schedule)
    assert all(same(a, b) for x in before for a, b in zip(before[x], captured.state()[x]))      # capturing runs nothing
    for t in (1, 2, 3, 70_001):
        schedule.copy_(corrections(t))
        graph.replay()
        eager.step(t)
        a, b = eager.state(), captured.state()
        assert all(same(x, y) for k in a for x, y in zip(a[k], b[k])), t


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_on_another_stream_behind_what_it_still_writes(eight):
    lists = Lists([300_000, 1000], eight=eight)
    want = Lists([300_000, 1000], eight=eight)
    for b in want.g:
        b.view.mul_(2.0)
    want.step(4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        for b in lists.g:
            b.view.mul_(2.0)
        lists.step(4)
    stream.synchronize()
    a, b = want.state(), lists.state()
    assert all(same(x, y) for k in a for x, y in zip(a[k], b[k]))


def test_what_the_betas_may_be():
    for beta1, beta2 in ((0.0, 0.0), (0.0, 0.9999), (0.999, 0.0)):
        lists = Lists([700])
        before = lists.state()
        lists.step(2, beta1=beta1, beta2=beta2)
        check(lists, before, lists.state(), 2, 0.1, beta1=beta1, beta2=beta2)


def test_a_gradient_may_be_used_twice():
    a, b = Lists([500, 500]), Lists([500, 500])
    a.g[1].view.copy_(a.g[0].view)
    b.g[1] = b.g[0]
    a.step(2), b.step(2)
    x, y = a.state(), b.state()
    assert all(same(p, q) for k in "pmv" for p, q in zip(x[k], y[k]))


def test_blocks_of_zeros_and_of_tiny_values():
    """A block whose largest value is below 2^-110 counts as zero, one above it does not; a v above zero keeps a code above zero."""
    lists = Lists([4 * BLOCK], eight=True, zeros=True)
    g = torch.zeros(4 * BLOCK)
    g[BLOCK] = 2.0 ** -40                                           # its square, times 1 - beta2: about 2^-90
    g[2 * BLOCK] = 2.0 ** -55                                       # 2^-120: m is held, v is not
    g[3 * BLOCK], g[3 * BLOCK + 1:] = 1.0, 2.0 ** -30               # v of the others 2^-60 of the largest: below the grid
    lists.g[0].view.copy_(g)
    before = lists.state()
    lists.step(1, 0.0)
    after = lists.state()
    check(lists, before, after, 1, 0.0)
    s, m, v = after["s"][0], after["m"][0], after["v"][0]
    assert (s[0] == 0).all() and s[1].all() and s[2, 0] > 0 and s[2, 1] == 0 and s[3].all()
    assert m[2 * BLOCK] == 0x7E and not v[2 * BLOCK:3 * BLOCK].any() and v[BLOCK] == 0x7B
    assert (v[3 * BLOCK + 1:] == 1).all()


def test_rounding_is_without_bias():
    """The mean of what 4096 blocks of one and the same content decode to, against the content: the mean of 4096 draws is off by
    5 sigma with a chance below 10^-6, sigma half a step at most."""
    blocks = 4096
    lists = Lists([blocks * BLOCK], eight=True, zeros=True)
    rng = np.random.default_rng(3)
    g = (rng.normal(0, 1, BLOCK) * 10.0 ** rng.uniform(-4, 0, BLOCK)).astype(np.float32)
    lists.g[0].view.copy_(torch.from_numpy(np.tile(g, blocks)))
    lists.step(1, 0.0)
    after = lists.state()
    m2, v2 = moments32(g, np.zeros(BLOCK, np.float32), np.zeros(BLOCK, np.float32), beta1=HYPER["beta1"], beta2=HYPER["beta2"])
    for codes, table, k, x in ((after["m"][0], E4M3, 0, m2), (after["v"][0], E5M2, 1, v2)):
        scale = after["s"][0][0, k]
        assert (after["s"][0][:, k] == scale).all()
        mean = decode(codes, table, scale).astype(np.float64).reshape(blocks, BLOCK).mean(0)
        y = np.abs(x) / scale
        low = np.minimum(np.searchsorted(table, y, side="right") - 1, table.size - 2)
        gap = (table[low + 1] - table[low]) * scale
        held = y >= table[1]                                        # below, v is held up
        assert (np.abs(mean - x) <= 5 * 0.5 * gap / math.sqrt(blocks) + 2.0 ** -16 * gap)[held].all()


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_offsets_beyond_32_bits(eight):
    """A tensor of more than 2^32 elements (states in 8 bits) or 2^31 (in 32): its ends and its middle, against the same values alone."""
    n = (1 << 32) + 700 if eight else (1 << 31) + 700
    if torch.cuda.mem_get_info()[0] < n * (7 if eight else 13):
        pytest.skip("not enough device memory")
    spots = [at // BLOCK * BLOCK for at in (0, n // 2, n - 4 * BLOCK)]
    small = Lists([4 * BLOCK - 5], BF16, BF16, eight=eight)
    blocks = -(-n // BLOCK)
    states = [(torch.uint8, n), (torch.uint8, n), (F32, 2 * blocks)] if eight else [(F32, n), (F32, n)]
    big = [torch.zeros(k, dtype=d, device="cuda") for d, k in [(BF16, n), (BF16, n), *states]]
    parts = [t[0] for t in small.tensors()]

    def cut(at):
        return [b[2 * at // BLOCK:][:a.numel()] if k == 4 else b[at:at + a.numel()].view(a.dtype) for k, (a, b) in enumerate(zip(parts, big))]

    for at in spots:
        for a, b in zip(parts, cut(at)):
            b.copy_(a)
    args = [[t] for t in big]
    # the draws depend on the block's place, so only what does not is compared: parameters, and scales
    (mqg.mqg_adamw8 if eight else mqg.mqg_adamw)(*args, 0.1, step=2, **HYPER, **({"seed": 7} if eight else {}))
    small.step(2)
    for at in spots:
        for k, (a, b) in enumerate(zip(parts, cut(at))):
            if eight and k in (2, 3):
                continue
            tail = 4 if k == 4 else 0                               # small's last block is short; big's is longer with zeros
            assert torch.equal(a[:a.numel() - tail], b[:a.numel() - tail]), (at, k)
    if eight:
        at = spots[1]
        codes = big[2][at:at + BLOCK].cpu().numpy()
        want = step8(np.zeros(BLOCK), small.state()["g"][0][:BLOCK], *[x[0][:BLOCK] for x in (Lists([4 * BLOCK - 5], BF16, BF16, eight=True).state()[c] for c in "mv")],
                     Lists([4 * BLOCK - 5], BF16, BF16, eight=True).state()["s"][0][:1], at // BLOCK, seed=7, step=2, decay=0.1, **HYPER)
        assert same(codes, want[2])
    untouched = big[0][4 * BLOCK:1 << 20]
    assert not untouched.any()


def test_what_the_binding_takes_and_refuses():
    t, eight = torch.zeros(300, device="cuda"), torch.zeros(300, dtype=torch.uint8, device="cuda")
    hyper = {**HYPER, "step": 1}
    assert mqg.mqg_adamw([], [], [], [], 0.1, **hyper) is None
    with pytest.raises(mqg.MqgError) as e:
        mqg.mqg_adamw([], [], [], [], [], **{**hyper, "lr": -1.0})
    assert e.value.status == mqg.MQG_ERR_INVALID
    with pytest.raises(mqg.MqgError, match="share memory"):
        mqg.mqg_adamw([t], [t.clone()], [t], [t.clone()], None, **hyper)
    with pytest.raises(TypeError, match="m.0. must be float32"):
        mqg.mqg_adamw([t], [t.clone()], [t.bfloat16()], [t.clone()], None, **hyper)
    with pytest.raises(ValueError, match="v.0. holds 299"):
        mqg.mqg_adamw([t], [t.clone()], [t.clone()], [t[:299].clone()], None, **hyper)
    with pytest.raises(ValueError, match="contiguous"):
        mqg.mqg_adamw([t], [torch.zeros(600, device="cuda")[::2]], [t.clone()], [t.clone()], None, **hyper)
    s = torch.zeros(4, device="cuda")
    with pytest.raises(TypeError, match="float8_e5m2"):
        mqg.mqg_adamw8([t], [t.clone()], [eight], [eight.clone().view(torch.float8_e4m3fn)], [s], None, seed=1, **hyper)
    with pytest.raises(ValueError, match="scales.0. holds 3"):
        mqg.mqg_adamw8([t], [t.clone()], [eight], [eight.clone()], [s[:3]], None, seed=1, **hyper)
    with pytest.raises(TypeError, match="factor must be float32"):
        mqg.mqg_adamw([t], [t.clone()], [t.clone()], [t.clone()], None, factor=t.double(), **hyper)
    # an iterator of tensors that nothing else holds
    mqg.mqg_adamw8(iter([t]), (torch.ones(300, device="cuda") for _ in range(1)), [eight], [eight.clone()], [s], iter([0.5]), seed=1,
                   **hyper)
    assert ((t + HYPER["lr"]).abs() <= 1e-3 * HYPER["lr"]).all()


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("types,shift", [((F32, F32), 0), ((BF16, BF16), 4), ((F32, BF16), 1)], ids=str)
def test_lists_that_give_a_warp_several_blocks(types, shift, eight):
    """More blocks than four times the warps that the device holds: whole runs of them, ends within a run, and tails."""
    sizes = [2_900_000, 1000, 2_000_000 + 37, 256 * 9, 0, 255, 256 * 32 + 1]
    lists = Lists(sizes, *types, eight=eight, shift=shift, seed=11)
    decays = [0.1 * (j % 2) for j in range(len(sizes))]
    before = lists.state()
    lists.step(3, decays, factor=torch.tensor([0.5], device="cuda"))
    after = lists.state()
    check(lists, before, after, 3, decays, k=0.5)
    lists.step(4, decays, factor=torch.tensor([math.nan], device="cuda"))
    again = lists.state()
    assert all(same(a, b) for x in after for a, b in zip(after[x], again[x]))


def test_a_nan_without_a_factor_stays_in_its_block():
    lists = Lists([3 * BLOCK, 40], eight=True)
    clean = Lists([3 * BLOCK, 40], eight=True)
    lists.g[0].view[BLOCK + 5] = math.nan
    lists.step(2), clean.step(2)
    a, b = lists.state(), clean.state()
    assert np.isnan(a["s"][0][1]).all() and np.isnan(a["p"][0][BLOCK + 5])
    other = np.r_[0:BLOCK, 2 * BLOCK:3 * BLOCK]
    for x in "pmv":
        assert same(a[x][0][other], b[x][0][other]) and same(a[x][1], b[x][1])
    assert np.isnan(a["p"][0]).sum() == 1 and same(a["s"][0][[0, 2]], b["s"][0][[0, 2]])


def test_decays_in_every_form():
    want = Lists([300, 20])
    want.step(2, [0.25, 0.5])
    for decays in (np.array([0.25, 0.5]), (0.25, 0.5), iter([0.25, 0.5])):
        lists = Lists([300, 20])
        lists.step(2, decays)
        assert all(same(a, b) for a, b in zip(want.state()["p"], lists.state()["p"]))
    same_for_all = [Lists([300, 20]) for _ in range(3)]
    for lists, decay in zip(same_for_all, (0.25, np.float32(0.25), [0.25, 0.25])):
        lists.step(2, decay)
    none = [Lists([300, 20]) for _ in range(2)]
    none[0].step(2, None), none[1].step(2, 0)
    for group in (same_for_all, none):
        assert all(same(a, b) for lists in group[1:] for a, b in zip(group[0].state()["p"], lists.state()["p"]))


FIRST_CALLS = """
import torch, paper_1804_08066_b200 as mqg
x = torch.randn({rows}, {dim}, device="cuda")
y, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty({rows}, 2, device="cuda")
w, dw, db = (torch.ones({dim}, device="cuda") for _ in range(3))
work = torch.empty(mqg.mqg_layer_norm_workspace_floats({rows}, {dim}), device="cuda")
t = [torch.zeros(300, device="cuda") for _ in range(4)]
s = torch.zeros(4, device="cuda")
codes = [torch.zeros(300, dtype=torch.uint8, device="cuda") for _ in range(2)]
hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    mqg.mqg_layer_norm(x, {rows}, {dim}, w, None, 1e-5, y, stats)
    mqg.mqg_layer_norm_grad(y, x, {rows}, {dim}, w, stats, dx, dw, db, work)
    mqg.mqg_adamw([t[0]], [t[1]], [t[2]], [t[3]], 0.0, **hyper)
    mqg.mqg_adamw8([t[0]], [t[1]], [codes[0]], [codes[1]], [s], 0.0, seed=1, **hyper)
t[1].fill_(1.0)
graph.replay()
torch.cuda.synchronize()
got = y.clone(), dx.clone(), dw.clone(), t[0].clone()
assert abs(float(y[0].mean())) < 1e-3 and (t[0] < -1.9e-3).all() and s[0] > 0
mqg.mqg_layer_norm(x, {rows}, {dim}, w, None, 1e-5, y, stats)
mqg.mqg_layer_norm_grad(y, x, {rows}, {dim}, w, stats, dx, dw, db, work)
assert torch.equal(got[0], y) and torch.equal(got[1], dx) and torch.equal(got[2], dw)
print("same")
"""


@pytest.mark.parametrize("rows,dim", [(40, 256), (3000, 1024), (500, 515), (60, 9000)])
def test_the_first_calls_of_a_process_may_be_captured(rows, dim):
    root = pathlib.Path(__file__).resolve().parent.parent
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS.format(rows=rows, dim=dim)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["same"], r.stderr[-2000:]


def test_zeros_of_either_sign_and_places_on_and_off_the_boundaries():
    """A gradient of zeros of both signs beside others, over steps that round small averages to zeros of either sign: the same bits
    wherever the tensors start."""
    results = []
    for shift in (0, 1, 3):
        lists = Lists([2 * BLOCK, 300], eight=True, zeros=True, shift=shift, seed=5)
        for t in range(1, 5):
            for b in lists.g:
                n = b.view.numel()
                i = torch.arange(n, device="cuda")
                b.view.copy_(torch.where(i % 3 == 0, torch.where(i % 2 == 0, 0.0, -0.0), (i % 7 - 3.0) * 10.0 ** (-(i % 9).float() - t % 2)))
            before = lists.state()
            lists.step(t, 0.0)
            check(lists, before, lists.state(), t, 0.0)
        results.append(lists.state())
    for other in results[1:]:
        assert all(same(a, b) for x in "pmvs" for a, b in zip(results[0][x], other[x]))
