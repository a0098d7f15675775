"""Device buffers with guard bytes around them, starting as far off a 16-byte boundary as a test wants."""
import torch

GUARD = 256
PATTERN = 0x5A


class Buffer:
    """`n` elements of `dtype`, `shift` elements behind a 256-byte boundary; filled from `values` or with the pattern."""

    def __init__(self, n, dtype, shift=0, values=None):
        size = torch.empty(0, dtype=dtype).element_size()
        self.before, self.bytes = GUARD + shift * size, n * size
        self.raw = torch.full((self.before + self.bytes + GUARD,), PATTERN, dtype=torch.uint8, device="cuda")
        # views of another type start at a multiple of its size in the storage: the allocation's first byte is one
        self.view = self.raw[self.before:self.before + self.bytes].view(dtype)
        if values is not None:
            self.view.copy_(values)

    def check(self):
        r = self.raw.cpu()
        assert (r[:self.before] == PATTERN).all(), "write before the buffer"
        assert (r[self.before + self.bytes:] == PATTERN).all(), "write past the buffer"

    def cpu(self):
        self.check()
        return self.view.cpu()


def same_bits(a, b):
    """Whether two CPU tensors of one floating type are equal bit for bit."""
    i = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return a.dtype == b.dtype and a.shape == b.shape and bool((a.contiguous().view(i) == b.contiguous().view(i)).all())
