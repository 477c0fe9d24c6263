"""GPU: halo_dropout against the 64-bit oracle.  The mask is compared exactly; a value is one product, with a residual also one sum,
each rounded to fp32 (u = 2^-24), the factor 1/(1-p) is rounded once, and a bf16 result is rounded once more (8 significant bits,
so 2^-8 of it): |err| <= 3 u |drop(x)| + u |y| (+ 2^-8 |y|, and half a step of the smallest numbers)."""
import numpy as np
import pytest
import torch

from oracle import adapters_oracle as orc
from paper_2501_02625_amd import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def padded(x, dtype, pad):
    """A device matrix of the values in a buffer with `pad` more columns of NaN, rows at a multiple of 16 bytes."""
    rows, cols = x.shape
    buf = torch.full((rows, (cols + pad + 7) // 8 * 8), float("nan"), dtype=dtype, device=gu.DEV)
    buf[:, :cols] = gu.to_dev(x).to(dtype)
    return buf[:, :cols]


@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 8, 0), (2, 7, 0), (3, 9, 8), (5, 4099, 5), (64, 512, 0), (257, 1000, 24),
                                           (1000, 24, 0), (33, 14336, 8), (7, 65537, 7)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_values(rows, cols, pad, dtype, residual, p):
    g = np.random.default_rng(rows * cols)
    seed, offset = int(g.integers(2**63)) * 2 + 1, int(g.integers(2**63)) * 2
    x = padded(g.standard_normal((rows, cols)).astype(np.float32), dtype, pad)
    res = padded(g.standard_normal((rows, cols)).astype(np.float32), dtype, pad) if residual else None
    room = torch.full((rows + 2, (cols + 7) // 8 * 8 + 16), 5.0, dtype=dtype, device=gu.DEV)
    out = room[1:rows + 1, 8:8 + cols]
    for y in (binding.halo_dropout(x, p, seed, offset, residual=res),
              binding.halo_dropout(x, p, seed, offset, residual=res, out=out)):
        d = orc.drop(x.double().cpu().numpy(), p, seed, offset)
        want = d if res is None else d + res.double().cpu().numpy()
        got = y.double().cpu().numpy()
        bound = 3 * U32 * np.abs(d) + (U32 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * np.abs(want) * (1 + 2.0 ** -8) + 1e-38
        bad = ~(np.abs(got - want) <= bound)
        assert y.dtype == dtype and not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3])
        if not residual:
            assert np.array_equal(got == 0, d == 0)
    out.fill_(5.0)
    assert (room == 5.0).all()


def test_dropped_elements_are_zero_whatever_they_were():
    x = torch.full((40, 200), float("inf"), device=gu.DEV)
    x[::2] = float("nan")
    y = binding.halo_dropout(x, 0.5, 3, 4)
    keep = gu.to_dev(orc.keep_mask(40, 200, 0.5, 3, 4))
    assert (y[~keep] == 0).all() and not torch.isfinite(y[keep]).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place_and_the_gradient(dtype):
    """The backward pass is the same call: <g, drop(x)> = <drop(g), x>, the mask being the same."""
    x = torch.randn(100, 136, device=gu.DEV).to(dtype)
    res = torch.randn(100, 136, device=gu.DEV).to(dtype)
    y = binding.halo_dropout(x, 0.3, 1, 2, residual=res)
    a, b = x.clone(), res.clone()
    assert torch.equal(binding.halo_dropout(a, 0.3, 1, 2, residual=res, out=a), y) and torch.equal(a, y)
    assert torch.equal(binding.halo_dropout(x, 0.3, 1, 2, residual=b, out=b), y)
    ones = torch.ones_like(x)
    grad = binding.halo_dropout(ones, 0.3, 1, 2)
    assert torch.equal(grad != 0, binding.halo_dropout(ones, 0.3, 1, 2, residual=None) != 0)
    # differences: drop is linear, element by element
    h = 0.5
    diff = (binding.halo_dropout(ones * (1 + h), 0.3, 1, 2).double() - binding.halo_dropout(ones * (1 - h), 0.3, 1, 2).double()) / (2 * h)
    assert (diff - grad.double()).abs().max() <= 2.0 ** (-7 if dtype == torch.bfloat16 else -22)
    assert not torch.equal(grad, binding.halo_dropout(ones, 0.3, 1, 3)) and not torch.equal(grad, binding.halo_dropout(ones, 0.3, 2, 2))


def test_a_row_that_is_taken_alone_or_with_others_has_the_mask_of_its_index():
    ones = torch.ones(64, 520, device=gu.DEV)
    whole = binding.halo_dropout(ones, 0.5, 9, 10)
    assert torch.equal(binding.halo_dropout(ones[:10], 0.5, 9, 10), whole[:10])
    assert torch.equal(binding.halo_dropout(ones[:, :136], 0.5, 9, 10), whole[:, :136])


def test_rows_beyond_32_bits():
    pitch = 1 << 27
    room = torch.zeros((39 * pitch + 64,), dtype=torch.bfloat16, device=gu.DEV)
    x = torch.as_strided(room, (40, 64), (pitch, 1))
    x.copy_(torch.randn(40, 64, device=gu.DEV))
    assert torch.equal(binding.halo_dropout(x, 0.2, 1, 1), binding.halo_dropout(x.contiguous(), 0.2, 1, 1))


def test_empty_and_refusals():
    x = torch.ones(4, 16, device=gu.DEV)
    assert binding.halo_dropout(x[:0], 0.1, 1, 1).shape == (0, 16)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(binding.HaloError) as e:
            binding.halo_dropout(x, p, 1, 1)
        assert e.value.status == binding.HALO_EINVAL
    with pytest.raises(TypeError):
        binding.halo_dropout(x.half(), 0.1, 1, 1)
    for kw in (dict(residual=x.bfloat16()), dict(residual=x[:2]), dict(out=x.t().contiguous().t())):
        with pytest.raises(AssertionError):
            binding.halo_dropout(x, 0.1, 1, 1, **kw)
    with pytest.raises(ValueError):
        binding.halo_dropout(x.cpu(), 0.1, 1, 1)
    with pytest.raises((OverflowError, TypeError)):
        binding.halo_dropout(x, 0.1, 2**64, 1)
