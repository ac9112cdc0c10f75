"""Rows for the tests of the operators around experts: any stride, any element to
start on, in a buffer whose other elements show whether something wrote there."""
import math

import torch

from paper_2409_02227_gb300 import goldy as G

TYPES = {"bf16": (torch.bfloat16, G.GOLDY_BF16), "f32": (torch.float32, G.GOLDY_F32)}
# a rounding's largest error relative to the value: half a step
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24                       # of an fp32 operation
GUARD = 776.0                        # 97 * 8: exact in bf16


class Rows:
    """rows x n elements in a larger buffer, `start` elements behind its
    beginning (a 16-byte boundary), rows `ld` apart."""

    def __init__(self, rows, n, dtype, ld=None, start=0, fill=None):
        self.ld = n if ld is None else ld
        self.start = start
        self.buffer = torch.full((start + max(1, rows) * self.ld + 64,), GUARD, device="cuda", dtype=dtype)
        self.t = self.buffer[start:start + max(1, rows) * self.ld].view(max(1, rows), self.ld)[:rows, :n]
        if fill is not None:
            self.t.copy_(fill)

    @property
    def ptr(self):
        return self.buffer.data_ptr() + self.start * self.buffer.element_size()

    def guarded(self):
        """Whether everything but the rows is as it was."""
        seen = self.buffer.clone()
        rows, n = self.t.shape
        seen[self.start:self.start + max(1, rows) * self.ld].view(max(1, rows), self.ld)[:rows, :n] = GUARD
        return bool((seen == GUARD).all())


def gen_of(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def workspace(need):
    """A workspace of exactly the asked size, in front of guarded memory."""
    return torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")


def within(got, ref, tol, what):
    """|got - ref| <= tol element by element; nothing but numbers."""
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - ref).abs() - tol
    if got.numel() and float(over.max()) > 0:
        at = int(over.flatten().argmax())
        raise AssertionError(f"{what}: {float(got.flatten()[at])} for {float(ref.flatten()[at])}, allowed "
                             f"{float(torch.as_tensor(tol, device=got.device).expand_as(got).flatten()[at]):.3e}")


def act64(z, act):
    """The activation in fp64."""
    if act == G.GOLDY_ACT_RELU:
        return z.clamp(min=0)
    if act == G.GOLDY_ACT_GELU:
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == G.GOLDY_ACT_GELU_TANH:
        return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == G.GOLDY_ACT_SILU:
        return z / (1.0 + torch.exp(-z))
    return z
