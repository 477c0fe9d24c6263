"""The root and the quotient inside halo_adamw are rounded to nearest, as its definition says: every significand of the root, quotients next to
the middle between two numbers, and both sides of the ranges in which the kernel leaves out what they do for extreme arguments.

With a gradient of 0, both betas 1/2 and a late step, m and v are halved, their corrections are 1, and with a rate of 1 and parameters of 0
the new parameter is -(m / (sqrt(v) + eps)), where nothing but the root, the sum and the quotient rounds."""
import numpy as np
import pytest
import torch

from paper_2501_02625_amd import binding
from tests.gpu_util import DEV, to_dev

pytestmark = pytest.mark.gpu
F = np.float32


def quotients(m, v, eps=0.0):
    """m / (sqrt(v) + eps) by the kernel: fp32 [n]."""
    double = lambda x: to_dev(x) * 2                                     # exact: the largest exponents here are far from the end
    p, g = torch.zeros(len(m), device=DEV), torch.zeros(len(m), device=DEV)
    m, v = double(m), double(v)
    half_m, half_v = m * 0.5, v * 0.5
    binding.halo_adamw([p], [g], [m], [v], step=200, lr=1.0, betas=(0.5, 0.5), eps=float(eps), weight_decay=0.0)
    assert torch.equal(m, half_m) and torch.equal(v, half_v)
    return -p.cpu().numpy()


def check(m, v, eps=0.0):
    with np.errstate(over="ignore", under="ignore", divide="ignore", invalid="ignore"):
        want = m / (np.sqrt(v) + F(eps))
    assert want.dtype == F
    got = quotients(m, v, eps)
    bad = np.flatnonzero(~((got == want) | (np.isnan(got) & np.isnan(want))))
    assert not len(bad), (len(bad), [(m[i], v[i], got[i], want[i]) for i in bad[:3]])


@pytest.mark.parametrize("exponent", [-99, -50, -1, 0, 1, 98])
def test_every_root(exponent):
    """Of all 2^23 significands at an even or odd exponent.  m is the root itself, so the quotient is 1 exactly if the kernel's root is that one: next
    to it, at r (1 + k), the quotient is 1 - k, and k is more than half a step of the numbers next to 1 on either side."""
    v = (np.arange(1 << 23, dtype=np.uint32) | np.uint32((127 + exponent) << 23)).view(F)
    r = np.sqrt(v.astype(np.float64)).astype(F)
    assert np.array_equal(r, np.sqrt(v))
    assert (quotients(r, v) == 1).all()


def significands(rng, n):
    return (rng.integers(0, 1 << 23, n).astype(np.uint32) | np.uint32(127 << 23)).view(F)


@pytest.mark.parametrize("at_m,at_d", [(0, 0), (30, -20), (-59, 49), (59, -49), (-59, -49), (59, 49)])
def test_quotients(at_m, at_d):
    """Random ones, and those whose exact value is next to the middle between two fp32 numbers: m = d (q + half a step) rounded.  A divisor d is
    the root of its square, rounded."""
    rng = np.random.default_rng(1)
    n = 1 << 21
    d, q = significands(rng, n), significands(rng, n)
    m = np.concatenate([significands(rng, n), (d.astype(np.float64) * (q.astype(np.float64) + 2.0 ** -24)).astype(F),
                        (d.astype(np.float64) * q).astype(F)])
    d = np.concatenate([d, d, d])
    v = d * d
    assert np.array_equal(np.sqrt(v), d)
    sign = np.where(rng.random(len(m)) < 0.5, F(-1), F(1))
    check(np.ldexp(m * sign, at_m).astype(F), np.ldexp(v, 2 * at_d).astype(F))


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -62, 2.0 ** -59, 1e-8, 2.0 ** 59, 2.0 ** 60, 2.0 ** 62])
def test_both_sides_of_the_inner_range(eps):
    """Groups of 4096 elements with v, m or both about the ends of the range (2^-100 and 2^100, 2^-60 and 2^60; the divisor's through eps), beyond
    them and at 0, and groups in which one element of many is."""
    rng = np.random.default_rng(2)
    ms, vs = [], []
    for at_v in (-126, -101, -100, -99, 0, 99, 100, 101, 125):
        for at_m in (-126, -61, -60, -59, 0, 59, 60, 61, 125):
            for alone in (False, True):
                m, v = np.ldexp(significands(rng, 4096), at_m).astype(F), np.ldexp(significands(rng, 4096), at_v).astype(F)
                if alone:
                    others = rng.random(4096) < 0.999
                    m[others], v[others] = significands(rng, others.sum()), significands(rng, others.sum())
                m[rng.random(4096) < 0.01] = 0
                v[rng.random(4096) < 0.01] = 0
                v[:2], m[:2] = np.ldexp(F(1), at_v), np.ldexp(F(1), at_m)
                ms.append(m)
                vs.append(v)
    check(np.concatenate(ms), np.concatenate(vs), eps)
