"""GPU: infinities and NaN in the operands of halo_adapters_* reach what the formulas say, as what the formulas say, and nothing else.

The inputs are such that T and S are exact (every row of X and E has one element that is not zero, a power of two): whatever way the
kernels take such a value into their matrix instructions, an infinite factor beside it gives an infinity, not NaN."""
import numpy as np
import pytest
import torch

from oracle import adapters_oracle as orc
from paper_2501_02625_amd import binding
from tests import gpu_util as gu
from tests.test_gpu_adapters import Case, U32, real, runs, scattered

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("b", [0, 5, 300, 1100])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_a_scale_of_an_adapter_without_tokens_is_not_used(value, b, p):
    """Its gradients are 0."""
    c = Case(b, 64, 136, 3, 24, [0, 2, -1, 2][:b] + [0] * (b - 4), ranks=[24, 17, 3], p=p)
    c.scale[1] = 1.0
    clean = c.run()
    c.scale[1] = value
    got = c.run()
    for x, y in zip(got, clean):
        assert torch.equal(x, y)
    assert not got[3][1].any() and not got[4][1].any()


@pytest.mark.parametrize("max_rank", [8, 16, 24, 64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
def test_an_infinite_scale_meets_the_adapters_own_rank_alone(max_rank, value):
    """An adapter of rank 1 in a pool that allots more: s T V^T has one term, an infinity of its sign."""
    c = Case(21, 72, 88, 2, max_rank, runs(21, 2, 4), ranks=[1, max_rank], base=True)
    c.scale[:] = 1.0
    clean = c.run()
    c.scale[0] = value
    Y, T, EX, GU, GV = c.run()
    mine = torch.from_numpy(c.of == 0).to(gu.DEV)
    assert torch.equal(Y[~mine], clean[0][~mine]) and torch.equal(EX[~mine], clean[2][~mine]) and torch.equal(T, clean[1])
    sign = lambda x: torch.sign(x) * np.sign(value) * float("inf")
    U, V = gu.bits_to_dev(c.U).float(), gu.bits_to_dev(c.V).float()
    assert torch.equal(Y[mine], sign(T[mine][:, :1] * V[0, :, 0]))
    E = gu.bits_to_dev(c.E)[mine].double()
    assert torch.equal(EX[mine], sign(((E @ V[0, :, :1].double()) * U[0, 0].double()).float()))


def product(a, b):
    """a [i, k], b [k, j]: the sum over k of every single product, as infinities and NaN go through it, and of its finite terms'
    absolute values."""
    with np.errstate(invalid="ignore"):
        terms = a[:, :, None] * b[None]
        return terms.sum(axis=1), np.where(np.isfinite(terms), np.abs(terms), 0.0).sum(axis=1)


def same(got, want, bound, what):
    g = got.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        ok = np.where(np.isfinite(want), np.abs(g - want) <= bound, np.where(np.isnan(want), np.isnan(g), g == want))
    assert g.shape == want.shape and ok.all(), (what, int((~ok).sum()), [(tuple(i), g[tuple(i)], want[tuple(i)]) for i in np.argwhere(~ok)[:4]])


def exact_case(b, m, n, rank, p):
    """X and E with one power of two a row, no element of U and V zero; two adapters, of which the second has a rank of its own."""
    c = Case(b, m, n, 2, rank, runs(b, 2, 3), ranks=[rank, max(1, rank - 5)], scale=False, p=p, base=True, seed=rank)
    g = np.random.default_rng(rank)
    for a, cols in (("X", m), ("E", n)):
        bits = np.zeros((b, cols), dtype=np.uint16)
        bits[np.arange(b), g.integers(0, cols, b)] = g.choice(np.array([0x3F80, 0xBF00, 0x4000, 0xC080], dtype=np.uint16), b)
        setattr(c, a, bits)
    return c


@pytest.mark.parametrize("where", ["U", "V", "X", "E", "T"])
@pytest.mark.parametrize("rank", [8, 16, 24, 64, 128])
@pytest.mark.parametrize("p", [0.0, 0.5])             # the factor of p = 0.5 is 2: no rounding
def test_infinities_are_what_the_formulas_say(where, rank, p):
    b, m, n = 21, 72, 88
    c = exact_case(b, m, n, rank, p)
    keep = orc.keep_mask(b, m, p, c.seed, c.offset)
    inf, ninf = 0x7F80, 0xFF80
    if where == "U":
        c.U[0, 2, 7], c.U[1, 0, 30] = inf, ninf
    elif where == "V":
        c.V[0, 5, 3], c.V[1, 60, 1] = ninf, inf
    elif where in "XE":
        bits = getattr(c, where)
        for t, value in ((1, inf), (4, ninf)):
            bits[t, np.flatnonzero(bits[t])[0]] = value
    X, E, U, V, of = *(gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V)), gu.to_dev(c.of)
    Y, T = binding.halo_adapters_fwd(X, U, V, of, base=c.dev_base(c.base_y), **c.kw())
    Tin = T.clone()
    if where == "T":
        Tin[0, 1], Tin[4, 0] = float("inf"), float("-inf")
    EX, GU, GV = binding.halo_adapters_bwd(E, X, Tin, U, V, of, base=c.dev_base(c.base_x), **c.kw())

    factor = 1.0 if p == 0.0 else 2.0
    x = np.where(keep, real(c.X) * factor, 0.0)
    e, u, v, t_in = real(c.E), real(c.U), real(c.V), Tin.double().cpu().numpy()
    for a in (0, 1):
        r, mine = int(c.ranks[a]), np.flatnonzero(c.of == a)
        part = lambda q: q[torch.from_numpy(mine).to(gu.DEV)]
        t = product(x[mine], u[a, :r].T)[0]
        same(part(T)[:, :r], t, 0.0, "T")                      # one term: exact
        low, size = product(t, v[a, :, :r].T)
        y = c.base_y[mine] + low
        same(part(Y), y, (44 + rank) * U32 * (size + np.abs(np.where(np.isfinite(y), y, 0.0))), "Y")
        s = product(e[mine], v[a, :, :r])[0]
        low, size = product(s, u[a, :r])
        low, size = np.where(keep[mine], low * factor, 0.0), size * factor
        ex = c.base_x[mine] + low
        same(part(EX), ex, (44 + rank) * U32 * (size + np.abs(np.where(np.isfinite(ex), ex, 0.0))), "EX")
        for got, (want, size), what in ((GU[a, :r], product(s.T, x[mine]), "GU"),
                                        (GV[a, :, :r], product(e[mine].T, t_in[mine, :r]), "GV")):
            same(got, want, (40 + b / 8) * U32 * size, what)


@pytest.mark.parametrize("rank", [16, 64])
@pytest.mark.parametrize("scale", [1.0, -1.5])
def test_zeros_of_either_sign(rank, scale):
    """-0 in T (S) is a zero like the other: nothing comes of it."""
    c = Case(33, 64, 72, 2, rank, scattered(33, 2), base=True)
    c.scale[:] = scale
    c.X[::3], c.E[1::3] = 0x8000, 0x8000
    X, E, U, V, of = *(gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V)), gu.to_dev(c.of)
    Y, T = binding.halo_adapters_fwd(X, U, V, of, base=c.dev_base(c.base_y), **c.kw())
    assert not T[::3].any() and torch.equal(Y[::3], c.dev_base(c.base_y)[::3])
    T[::3] = -0.0
    EX, GU, GV = binding.halo_adapters_bwd(E, X, T, U, V, of, base=c.dev_base(c.base_x), **c.kw())
    assert torch.equal(EX[1::3], c.dev_base(c.base_x)[1::3])
    c.check(Y, T, EX, GU, GV)


@pytest.mark.parametrize("rank", [16, 64])
@pytest.mark.parametrize("power", [60, 100, 118])
def test_small_thin_values(rank, power):
    """T of about 2^-power meets V of about 2^(power - 20): pieces of T are lost below 2^-133 only."""
    b, m, n = 18, 64, 72
    c = Case(b, m, n, 2, rank, runs(b, 2, 3), scale=False, base=False, seed=power)
    g = np.random.default_rng(power)
    bits = lambda *shape, std: (np.frombuffer((g.standard_normal(shape) * std).astype(np.float32).tobytes(), dtype=np.uint32) >> 16) \
        .astype(np.uint16).reshape(shape)
    c.U, c.V = bits(2, rank, m, std=2.0 ** -power), bits(2, n, rank, std=2.0 ** (power - 20))
    X, U, V, of = *(gu.bits_to_dev(a) for a in (c.X, c.U, c.V)), gu.to_dev(c.of)
    Y, T = binding.halo_adapters_fwd(X, U, V, of, **c.kw())
    t = T.cpu().numpy().astype(np.float64)
    for a in (0, 1):
        mine = np.flatnonzero(c.of == a)
        want, size = product(t[mine], real(c.V[a]).T)
        bound = (44 + rank) * U32 * size + rank * 2.0 ** -133 * np.abs(real(c.V[a])).max()
        same(Y[torch.from_numpy(mine).to(gu.DEV)], want, bound, "Y")
