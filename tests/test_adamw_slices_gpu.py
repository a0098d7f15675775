"""AdamW over tensors that are slices of shared storages: in and out of order, empty ones among them, views of two types of one storage."""
import numpy as np
import pytest
import torch

import paper_1804_08066_b200 as mqg

from .test_adamw_gpu import HYPER, Lists, check, same

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SIZES = [0, 300, 5, 0, 1024, 7, 513, 0, 64, 2049, 0]


class Slice:
    """A slice of a storage in the place of a buffer of its own."""

    def __init__(self, view):
        self.view = view

    def cpu(self):
        return self.view.cpu()


def slices_of(buffers, order, lead):
    """The buffers' contents as slices of one vector that begins with `lead` other elements, laid out in the given order."""
    kind = buffers[0].view.dtype
    raw = torch.uint8 if kind.itemsize == 1 else kind
    flat = torch.zeros(lead + sum(b.view.numel() for b in buffers), dtype=raw, device="cuda").view(kind)
    at, out = lead, [None] * len(buffers)
    for j in order:
        n = buffers[j].view.numel()
        flat.view(raw)[at:at + n].copy_(buffers[j].view.view(raw))
        out[j] = Slice(flat[at:at + n])
        at += n
    return out


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, BF16)], ids=str)
@pytest.mark.parametrize("lead", [0, 1, 4])
@pytest.mark.parametrize("order", ["first to last", "last to first", "mixed"])
def test_slices_of_one_vector_each(order, lead, types, eight):
    places = {"first to last": list(range(len(SIZES))), "last to first": list(range(len(SIZES)))[::-1],
              "mixed": np.random.default_rng(1).permutation(len(SIZES)).tolist()}[order]
    lists = Lists(SIZES, *types, eight=eight, seed=3)
    for name in "pgmvs":
        if getattr(lists, name):
            setattr(lists, name, slices_of(getattr(lists, name), places, lead))
    for t in (1, 2):
        before = lists.state()
        lists.step(t, 0.1)
        check(lists, before, lists.state(), t, 0.1)


def test_views_of_two_types_of_one_storage():
    """Parameters in fp32 and bf16, gradients, m and v side by side in one allocation of bytes."""
    sizes = [200, 36, 512, 8, 1000]
    made = {BF16: Lists(sizes, BF16, BF16, seed=4), F32: Lists(sizes, F32, F32, seed=4)}
    lists = Lists(sizes, F32, F32, seed=4)
    memory = torch.zeros(sum(16 * n + 64 for n in sizes), dtype=torch.uint8, device="cuda")
    at = 0
    for j in range(len(sizes)):
        kind = (F32, BF16)[j % 2]
        for name in "pgmv":
            source = getattr(made[kind], name)[j].view
            size = source.numel() * source.element_size()
            view = memory[at:at + size].view(source.dtype)
            view.copy_(source)
            getattr(lists, name)[j] = Slice(view)
            at += -(-size // 4) * 4
    before = lists.state()
    lists.step(7, 0.1)
    check(lists, before, lists.state(), 7, 0.1)


def test_scales_of_every_block_of_a_tensor_beyond_32_bits():
    """Scales of three places of a tensor of more than 2^32 elements, all but the short last block's."""
    n, block = (1 << 32) + 700, 256
    if torch.cuda.mem_get_info()[0] < 7 * n:
        pytest.skip("not enough device memory")
    held = 4 * block - 5
    small = Lists([held], BF16, BF16, eight=True, seed=6)
    big = [torch.zeros(n, dtype=d, device="cuda") for d in (BF16, BF16, torch.uint8, torch.uint8)]
    scales = torch.zeros(2 * -(-n // block), device="cuda")
    spots = [at // block * block for at in (0, n // 2, n - 4 * block)]
    parts = [t[0] for t in small.tensors()]
    for at in spots:
        for a, b in zip(parts, big):
            b[at:at + held].view(a.dtype).copy_(a)
        scales[2 * at // block:][:8].copy_(parts[4])
    mqg.mqg_adamw8(*[[t] for t in (*big, scales)], 0.1, step=2, seed=7, **HYPER)
    small.step(2)
    want = small.state()["s"][0].reshape(-1)
    for at in spots:
        assert same(scales[2 * at // block:][:6].cpu().numpy(), want[:6])
