"""AdamW's parameter step where the root's argument or the divisor leaves what an ordinary step meets: averages below fp32's smallest
normal number beside the smallest eps, divisors near fp32's largest number."""
import numpy as np
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .adamw_plain import moments32
from .buffers import Buffer

pytestmark = pytest.mark.gpu

f32 = np.float32
U = 2.0 ** -24


def step(g, v, eight, shift, schedule=None, **hyper):
    """Parameters after one step from zeros, m = 0, v as given (zeros in 8 bits)."""
    n = g.size
    p, grads = Buffer(n, torch.float32, shift, torch.zeros(n)), Buffer(n, torch.float32, shift, torch.from_numpy(g))
    if eight:
        assert not v.any()
        m, vv = (Buffer(n, torch.uint8, shift, torch.zeros(n, dtype=torch.uint8)) for _ in range(2))
        scales = torch.zeros(mqg.mqg_adamw8_scale_floats(n), device="cuda")
        mqg.mqg_adamw8([p.view], [grads.view], [m.view], [vv.view], [scales], None, seed=3, schedule=schedule, **hyper)
    else:
        m, vv = Buffer(n, torch.float32, shift, torch.zeros(n)), Buffer(n, torch.float32, shift, torch.from_numpy(v))
        mqg.mqg_adamw([p.view], [grads.view], [m.view], [vv.view], None, schedule=schedule, **hyper)
    return p.cpu().double().numpy()


def check(got, g, v, *, lr, beta1, beta2, eps, step, c1=None, c2=None):
    m2, v2 = moments32(g, np.zeros_like(g), v, beta1=beta1, beta2=beta2)
    c1, c2 = 1 - beta1 ** step if c1 is None else c1, 1 - beta2 ** step if c2 is None else c2
    term = lr / c1 * (m2.astype(np.float64) / (np.sqrt(v2.astype(np.float64)) / np.sqrt(c2) + eps))
    # Roundings of 2^-24 each: a 3 (lr's own, c1, the quotient); r2 2.5 (c2 halved, the root, the quotient); the root 4 and the quotient 4
    # (two units in the last place); a root of zero where d has nothing of it 0.5; d's product, eps's own, d's sum; the last
    # product and the difference: 19.  The parameter's subnormal numbers do not occur.
    assert (np.abs(term) > 1e-30).all() and (np.abs(term) < 1e38).all()
    assert (np.abs(got + term) <= 19 * U * np.abs(term)).all(), np.max(np.abs(got + term) / np.abs(term)) / U


def gradients(n, size, seed):
    rng = np.random.default_rng(seed)
    return (rng.choice([-1.0, 1.0], n) * size * 10.0 ** rng.uniform(-0.5, 0.5, n)).astype(f32)


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("eps", [2.0 ** -50, 1e-12, 1e-8])
@pytest.mark.parametrize("beta2", [0.99, 0.9999, 1 - 2.0 ** -20])
def test_averages_below_the_smallest_normal_number(beta2, eps, shift, eight):
    g = gradients(700, 1e-17 if beta2 > 0.9999 else 1e-19, 1)
    hyper = dict(lr=1.0, beta1=0.9, beta2=beta2, eps=eps, step=1)
    v = np.zeros_like(g)
    _, v2 = moments32(g, v, v, beta1=0.9, beta2=beta2)
    assert (v2 < 2.0 ** -126).all() and v2.any()
    check(step(g, v, eight, shift, **hyper), g, v, **hyper)


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("eps", [2.0 ** 60, 2.0 ** 64, 2.0 ** 76, 1e30, 2.0 ** 126, 1.5 * 2.0 ** 126, 2e38, 3.3e38])
def test_the_largest_eps(eps, shift, eight):
    g = gradients(700, 1e17, 2)
    v = np.zeros_like(g)
    hyper = dict(lr=1e25, beta1=0.9, beta2=0.999, eps=eps, step=2)
    check(step(g, v, eight, shift, **hyper), g, v, **{**hyper, "eps": float(f32(eps))})


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("exponent", [-30, -100, -126, -149])
def test_a_schedule_with_the_smallest_correction(exponent, shift):
    """1 - b2^t as a program that makes it up may pass it: 2^exponent."""
    g = gradients(700, 1e17, 3)
    v = np.full(700, 2.0 ** 104, f32)
    lr, c2 = float(f32(1e38)), 2.0 ** exponent
    schedule = torch.tensor([lr, 0.5, c2, 5.0], dtype=torch.float64).float()
    assert float(schedule[2]) == c2
    hyper = dict(beta1=0.9, beta2=0.999, eps=1e-8, step=0)
    got = step(g, v, False, shift, schedule=schedule.cuda(), lr=0.25, **hyper)
    keep = np.full(700, True)
    check(got[keep], g, v, lr=lr, c1=0.5, c2=c2, **{**hyper, "step": 5})


def test_averages_that_overflow():
    """v' beyond fp32's range: its root is infinite, and the quotient zero."""
    g = gradients(300, 1e25, 4)
    for eps in (2.0 ** -50, 1e-8, 3e38):
        for shift in (0, 1):
            got = step(g, np.zeros_like(g), False, shift, lr=1.0, beta1=0.9, beta2=0.999, eps=eps, step=1)
            assert not got.any()
