"""Inputs and bounds for the tests of what stands around a layer's products.

u = 2^-24 is half a step of fp32 next to 1.  A sum of n numbers added one after another is off by at most n u times the sum of their
magnitudes; kernels add at most n / 64 + 32 of a row after another (at least 64 lanes share it, then the lanes' sums meet), and at most n / 16 +
64 of a column."""
import numpy as np
import torch

from tests.gpu_util import DEV

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.bfloat16, torch.float32]


def host(t):
    return t.detach().double().cpu().numpy()


def matrix(values, dtype, extra=0):
    """The values in a buffer whose rows begin at multiples of 16 bytes; what lies between the rows is NaN."""
    v = torch.as_tensor(np.asarray(values)).to(dtype)
    rows, cols = v.shape
    per16 = 16 // v.element_size()
    pitch = (-(-cols // per16) + extra) * per16
    buffer = torch.full((rows, max(pitch, per16)), float("nan"), dtype=dtype, device=DEV)
    m = buffer[:, :cols]
    m.copy_(v.to(DEV))
    return m


def target(rows, cols, dtype, extra=1):
    """An output in a wider buffer, and a check that nothing but it was written."""
    per16 = 16 // torch.empty((), dtype=dtype).element_size()
    pitch = (-(-cols // per16) + extra) * per16
    buffer = torch.full((rows + 2, pitch), 7.5, dtype=dtype, device=DEV)

    def untouched():
        rest = buffer.clone()
        rest[1:rows + 1, :cols] = 7.5
        return bool((rest == 7.5).all())

    return buffer[1:rows + 1, :cols], untouched


def row_terms(n):
    return n / 64 + 32


def column_terms(n):
    return min(n, n / 16 + 64) + 8


def within(got, want, bound, what):
    g = host(got) if isinstance(got, torch.Tensor) else np.asarray(got, np.float64)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bad = ~(np.abs(g - want) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d off, first at %s: got %r want %r bound %r"
                             % (what, bad.sum(), bad.size, i, g[i], want[i], np.broadcast_to(bound, g.shape)[i]))


def act_bound(z, y, name, dtype=torch.float32):
    """How far act(z) may be from its value y: the exponential's argument is off by a few roundings, which counts where it is large and
    negative; the reciprocal, the exponential and the products by one rounding each (1.5 for the polynomial of gelu).  For bf16 results
    gelu's polynomial is a shorter one, 3.2e-5 of the tail Phi(-|z|) off at most: z times the tail is all of y for z < 0, and at most y for
    z > 0, where y = z (1 - tail) and tail <= 1/2."""
    z, y = np.asarray(z), np.abs(y)
    below = z < 0
    if name in ("none", "relu"):
        return 0.0 * y
    if name == "silu":
        return (np.abs(z) * below + 10) * U * y + 1e-30
    if name == "gelu":
        return ((z * z * below + 20) * U + (3.2e-5 if dtype == torch.bfloat16 else 0.0)) * y + 1e-30
    return (5 * np.abs(1.6 * (z + 0.044715 * z ** 3)) * below + 14) * U * y + 1e-30


SLOPE = 24 * U          # of act': two terms of at most 1.13, each a product of up to six rounded factors
