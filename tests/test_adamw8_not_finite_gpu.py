"""States in 8 bits whose blocks hold infinities and NaN, from gradients or from the codes themselves: the same bits on and off the
boundaries of four elements, and each code's value as its format has it."""
import math

import numpy as np
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .buffers import Buffer

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
F32, BF16 = torch.float32, torch.bfloat16
BLOCKS = 6


class Tensor:
    def __init__(self, p, g, m, v, s, kinds, shift):
        n = p.numel()
        self.p, self.g = Buffer(n, kinds[0], shift, p.to(kinds[0])), Buffer(n, kinds[1], shift, g.to(kinds[1]))
        self.m, self.v = Buffer(n, torch.uint8, shift, m), Buffer(n, torch.uint8, shift, v)
        self.s = Buffer(s.numel(), F32, shift, s)

    def step(self, t, **more):
        mqg.mqg_adamw8([self.p.view], [self.g.view], [self.m.view], [self.v.view], [self.s.view], 0.1, step=t, seed=11, **{**HYPER, **more})

    def state(self):
        return [b.cpu() for b in (self.p, self.m, self.v, self.s)]


def alike(a, b):
    """The same bits, NaN of parameters apart."""
    for x, y in zip(a, b):
        if x.dtype != torch.uint8:
            x, y = x.float(), y.float()
            assert torch.equal(x.isnan(), y.isnan())
            x, y = x.nan_to_num(7.0).view(torch.int32), y.nan_to_num(7.0).view(torch.int32)
        assert torch.equal(x, y), (x != y).nonzero().flatten()[:8]


def ordinary(seed):
    gen = torch.Generator().manual_seed(seed)
    n = BLOCKS * 256 + 37
    p, g = torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    m = torch.randint(0, 0x7F, (n,), generator=gen) | torch.randint(0, 2, (n,), generator=gen) << 7
    v = torch.randint(0x30, 0x7C, (n,), generator=gen)
    s = (torch.rand(2 * (BLOCKS + 1), generator=gen) + 0.5) * torch.tensor([1 / 448, 1 / 57344]).repeat(BLOCKS + 1)
    return p, g, m.to(torch.uint8), v.to(torch.uint8), s


KINDS = pytest.mark.parametrize("kinds", [(F32, F32), (F32, BF16), (BF16, BF16)], ids=str)


@KINDS
def test_gradients_that_overflow(kinds):
    """Blocks with an infinite m' and v', of either sign; with an infinite v' alone; with a NaN; then steps from what they left."""
    p, g, m, v, s = ordinary(1)
    g[3], g[100] = 3e38, -3e38                                       # times 4: infinities
    g[256 + 7] = -3e38
    g[2 * 256 + 9] = 1e25                                           # its square only
    g[3 * 256 + 200] = math.nan
    g[-1] = 3e38
    tensors = [Tensor(p, g, m, v, s, kinds, shift) for shift in (0, 1, 2, 3, 5)]
    for t in (1, 2, 3):
        for x in tensors:
            x.step(t, grad_scale=4.0)
        for x in tensors[1:]:
            alike(tensors[0].state(), x.state())
        if t == 1:
            _, mc, vc, sc = tensors[0].state()
            assert torch.equal(sc[:4].isinf(), torch.tensor([True] * 4)) and sc[4].isfinite() and sc[5].isinf()
            assert sc[6:8].isnan().all() and sc[8:12].isfinite().all() and sc[12:].isinf().all()
        for x in tensors:
            x.g.view.copy_(torch.randn(p.numel(), generator=torch.Generator().manual_seed(t)).to(kinds[1]))


@KINDS
def test_every_code_is_read_as_its_format_has_it(kinds):
    """All 256 codes of m, the 128 of v, finite or not, in blocks of their own: a step with b1 = b2 = 1 - 2^-24 and no gradient leaves
    their values as they are, seen in the blocks' scales (m's and v's largest) and in the parameters."""
    codes = torch.arange(256).to(torch.uint8)
    n = 256 * 256
    scale = torch.tensor([1.0, 1.0]).repeat(256)
    states = []
    for shift in (0, 1, 2, 3, 6):
        m = codes.repeat_interleave(256)
        v = (codes & 0x7F).repeat_interleave(256)
        x = Tensor(torch.ones(n), torch.zeros(n), m, v, scale, kinds, shift)
        x.step(1, beta1=1 - 2.0 ** -24, beta2=1 - 2.0 ** -24)
        states.append(x.state())
    for other in states[1:]:
        alike(states[0], other)
    left = states[0][3].view(256, 2).double()
    for k, kind, top in ((0, torch.float8_e4m3fn, 448.0), (1, torch.float8_e5m2, 57344.0)):
        want = (codes if k == 0 else codes & 0x7F).view(kind).float().double().abs() / top
        finite = want.isfinite()
        # b x: one rounding and b's distance from 1; the division by the largest: one more
        assert ((left[:, k] - want).abs() <= 4 * 2.0 ** -24 * want)[finite].all()
        assert torch.equal(left[:, k].isnan(), want.isnan()) and torch.equal(left[:, k].isinf(), want.isinf())


def test_special_codes_among_others():
    p, g, m, v, s = ordinary(2)
    m[5], m[256 + 6] = 0x7F, 0xFF
    v[2 * 256 + 7], v[3 * 256 + 8], v[4 * 256 + 9] = 0x7C, 0x7D, 0x7F
    m[-1], v[-2] = 0xFF, 0x7C
    tensors = [Tensor(p, g, m, v, s, (F32, F32), shift) for shift in (0, 1, 2, 7)]
    for t in (4, 5):
        for x in tensors:
            x.step(t)
        for x in tensors[1:]:
            alike(tensors[0].state(), x.state())
    assert np.isnan(tensors[0].state()[0].numpy()).sum() > 0
