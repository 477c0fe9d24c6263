"""halo_layer_norm_fwd and halo_layer_norm_bwd against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as orc
from paper_2501_02625_amd import binding
from tests.around_util import DTYPES, HALF, U, column_terms, host, matrix, row_terms, target, within
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
KINDS = ["layer", "rms"]
COLS = [1, 2, 7, 8, 9, 63, 64, 255, 512, 513, 1000, 1024, 1025, 2048, 2049, 4096, 4099, 8192, 8200, 14336, 16384, 16385, 32767, 32768]


def inputs(rows, cols, dtype, wdtype, seed, bias=True, shift=0.3):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, cols)) + shift
    x[:, rng.integers(0, cols, max(1, cols // 1000))] *= 50.0
    w = torch.tensor(1 + 0.2 * rng.normal(size=cols)).to(wdtype).to(DEV)
    b = torch.tensor(0.2 * rng.normal(size=cols)).to(wdtype).to(DEV) if bias else None
    return matrix(x, dtype, extra=seed % 2), w, b, rng


def check_fwd(x, w, b, eps, kind, y, mean, rstd, what):
    X, W, B = host(x), host(w) if w is not None else None, host(b) if b is not None else None
    want, m, r = orc.norm(X, W, B, eps, kind)
    k = row_terms(X.shape[1])
    off_mean = k * U * np.abs(X).mean(axis=1) if kind == "layer" else 0.0 * m
    # of rstd, relative: the sum of squares, the division, sum, root and reciprocal, and what a mean that is off adds
    off_rstd = (k / 2 + 6) * U + (off_mean * r) ** 2
    if mean is not None:
        within(mean, m, off_mean + U * np.abs(m), what + " mean")
    if rstd is not None:
        within(rstd, r, 2 * off_rstd * r, what + " rstd")
    aw = 1.0 if W is None else np.abs(W)
    centred = np.abs(want - (0.0 if B is None else B))
    bound = aw * (off_mean * r)[:, None] * 2 + centred * (2 * off_rstd[:, None] + 4 * U) + U * np.abs(want) + HALF[x.dtype] * np.abs(want)
    within(y, want, bound, what + " Y")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_fwd(cols, dtype, kind):
    for rows in (1, 5):
        x, w, b, _ = inputs(rows, cols, dtype, DTYPES[cols % 2], cols + rows, bias=cols % 3 > 0)
        out, untouched = target(rows, cols, dtype)
        y, mean, rstd = binding.halo_layer_norm_fwd(x, w, b, eps=1e-5, kind=kind, Y=out)
        assert y is out and untouched() and (mean is None) == (kind == "rms")
        check_fwd(x, w, b, 1e-5, kind, y, mean, rstd, "%d x %d" % (rows, cols))


@pytest.mark.parametrize("rows,cols", [(1000, 64), (4097, 128), (257, 1000), (64, 4096), (70001, 40), (513, 8192), (300, 20000)])
def test_fwd_many_rows(rows, cols):
    x, w, b, _ = inputs(rows, cols, torch.bfloat16, torch.float32, 3)
    y, mean, rstd = binding.halo_layer_norm_fwd(x, w, b, eps=1e-6)
    check_fwd(x, w, b, 1e-6, "layer", y, mean, rstd, "%d x %d" % (rows, cols))


@pytest.mark.parametrize("dtype", DTYPES)
def test_fwd_without(dtype):
    """No weight, no bias, no statistics; statistics given; in place."""
    x, w, b, _ = inputs(9, 1003, dtype, dtype, 4)
    y, mean, rstd = binding.halo_layer_norm_fwd(x, want_stats=False)
    assert mean is None and rstd is None
    check_fwd(x, None, None, 1e-5, "layer", y, None, None, "plain")
    m, r = torch.full((2, 9), 3.0, device=DEV)
    z, m2, r2 = binding.halo_layer_norm_fwd(x, w, b, mean=m, rstd=r)
    assert m2.data_ptr() == m.data_ptr() and r2.data_ptr() == r.data_ptr()
    copy = matrix(x.float().cpu().numpy(), dtype)
    binding.halo_layer_norm_fwd(copy, w, b, Y=copy)
    assert torch.equal(copy, z)
    only_bias, _, _ = binding.halo_layer_norm_fwd(x, None, b)
    check_fwd(x, None, b, 1e-5, "layer", only_bias, None, None, "bias")


@pytest.mark.parametrize("kind", KINDS)
def test_fwd_of_constant_rows_and_zeros(kind):
    """Nothing to divide by but eps; a mean far from 0, where the squares of the values themselves would cancel."""
    x = matrix(np.stack([np.zeros(1000), np.full(1000, 300.0), 1e4 + np.arange(1000) % 2]), torch.float32)
    y, mean, rstd = binding.halo_layer_norm_fwd(x, kind=kind, eps=1e-3)
    check_fwd(x, None, None, 1e-3, kind, y, mean, rstd, "constant")


def test_fwd_eps_zero_of_a_zero_row_is_nan():
    y, _, rstd = binding.halo_layer_norm_fwd(torch.zeros(2, 16, device=DEV), eps=0.0)
    assert torch.isnan(y).all() and torch.isinf(rstd).all()


def test_fwd_nonfinite_rows_stay_rows():
    x, w, b, _ = inputs(6, 777, torch.float32, torch.float32, 5)
    clean, _, _ = binding.halo_layer_norm_fwd(x, w, b)
    x[2, 5], x[4, 776] = float("inf"), float("nan")
    y, _, _ = binding.halo_layer_norm_fwd(x, w, b)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[[2, 4]]).all()


def check_bwd(e, x, mean, rstd, w, base, kind, ex, gw, gb, what):
    E, X, M, R = host(e), host(x), host(mean) if mean is not None else None, host(rstd)
    W = host(w) if w is not None else None
    want, ww, wb = orc.norm_grad(E, X, M, R, W, host(base) if base is not None else None, kind)
    rows, cols = E.shape
    k, c = row_terms(cols), column_terms(rows)
    xh = (X - (M[:, None] if kind == "layer" else 0.0)) * R[:, None]
    d = np.abs(E * (1.0 if W is None else W))
    mean_d = d.mean(axis=1, keepdims=True) if kind == "layer" else 0.0
    mean_dx = (d * np.abs(xh)).mean(axis=1, keepdims=True)
    if ex is not None:
        bound = R[:, None] * (8 * U * d + (k + 10) * U * mean_d + np.abs(xh) * (k + 14) * U * mean_dx) + 2 * U * np.abs(want)
        if base is not None:
            bound = bound + 2 * U * np.abs(host(base))
        within(ex, want, bound + HALF[e.dtype] * np.abs(want), what + " EX")
    if gw is not None:
        within(gw, ww, (c + 4) * U * (np.abs(E) * np.abs(xh)).sum(axis=0), what + " GW")
    if gb is not None:
        within(gb, wb, c * U * np.abs(E).sum(axis=0), what + " GB")


def saved(x, kind, eps=1e-5):
    _, m, r = orc.norm(host(x), None, None, eps, kind)
    f = lambda v: torch.tensor(v, dtype=torch.float32, device=DEV)
    return (f(m) if kind == "layer" else None), f(r)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_bwd(cols, dtype, kind):
    for rows in (1, 37):
        x, w, _, rng = inputs(rows, cols, dtype, DTYPES[cols % 2], cols + rows)
        e = matrix(rng.normal(size=(rows, cols)), dtype, extra=1)
        base = matrix(rng.normal(size=(rows, cols)), dtype) if cols % 3 else None
        mean, rstd = saved(x, kind)
        out, untouched = target(rows, cols, dtype)
        ex, gw, gb = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind=kind, base=base, EX=out)
        assert untouched()
        check_bwd(e, x, mean, rstd, w, base, kind, ex, gw, gb, "%d x %d" % (rows, cols))


@pytest.mark.parametrize("rows,cols", [(1000, 64), (4097, 128), (2051, 1000), (640, 4096), (70001, 40), (513, 8192), (300, 20000), (1100, 32768)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_bwd_many_rows(rows, cols, dtype):
    x, w, _, rng = inputs(rows, cols, dtype, torch.float32, 3)
    e, base = (matrix(rng.normal(size=(rows, cols)), dtype) for _ in range(2))
    mean, rstd = saved(x, "layer")
    ex, gw, gb = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base)
    check_bwd(e, x, mean, rstd, w, base, "layer", ex, gw, gb, "%d x %d" % (rows, cols))


@pytest.mark.parametrize("cols", [40, 1003, 4096, 20000])
def test_bwd_each_output_alone(cols):
    """The same numbers, whichever outputs are wanted; EX in E and in base; a second call on the same workspace."""
    x, w, _, rng = inputs(200, cols, torch.bfloat16, torch.bfloat16, 6)
    e, base = (matrix(rng.normal(size=(200, cols)), torch.bfloat16) for _ in range(2))
    mean, rstd = saved(x, "layer")
    whole = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device=DEV)
    for want in range(1, 8):
        names = dict(want_ex=bool(want & 1), want_gw=bool(want & 2), want_gb=bool(want & 4))
        got = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base, workspace=ws, **names)
        for k in range(3):
            assert (got[k] is None) == (not want >> k & 1)
            assert got[k] is None or torch.equal(got[k], whole[k])
    for place in (0, 1):
        e2, b2 = (matrix(t.float().cpu().numpy(), torch.bfloat16) for t in (e, base))
        got = binding.halo_layer_norm_bwd(e2, x, mean, rstd, w, base=b2, EX=(e2, b2)[place])
        assert all(torch.equal(a, b) for a, b in zip(got, whole))
    gb_only = binding.halo_layer_norm_bwd(e, None, None, None, None, want_ex=False, want_gw=False)[2]
    assert torch.equal(gb_only, whole[2])


def test_bwd_of_no_rows():
    e = torch.empty(0, 100, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(100, device=DEV)
    nothing = torch.empty(0, device=DEV)
    ones = lambda: torch.ones(100, device=DEV)
    ex, gw, gb = binding.halo_layer_norm_bwd(e, e, nothing, nothing, w, GW=ones(), GB=ones())
    assert ex.shape == (0, 100) and not gw.any() and not gb.any()
    assert binding.halo_layer_norm_fwd(e, w)[0].shape == (0, 100)


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_are_those_of_the_forward_pass(kind):
    """sum(E y) along a direction of X and along one of weight and bias, by differences of the oracle in 64 bits: five points 1e-4 apart, off
    by about h^4 of the fifth derivative, and in the weight y is linear.  1e-5: 100 roundings of fp32 in a row of 50."""
    x, w, b, rng = inputs(3, 50, torch.float32, torch.float32, 8, shift=0.0)
    E, D = rng.normal(size=(3, 50)), rng.normal(size=(3, 50))
    y, mean, rstd = binding.halo_layer_norm_fwd(x, w, b, kind=kind)
    ex, gw, gb = binding.halo_layer_norm_bwd(matrix(E, torch.float32), x, mean, rstd, w, kind=kind)
    h = 1e-4
    f = lambda t: (orc.norm(host(x) + t * D, host(w), host(b), 1e-5, kind)[0] * E).sum()
    want = (8 * (f(h) - f(-h)) - (f(2 * h) - f(-2 * h))) / (12 * h)
    scale = np.abs(host(ex) * D).sum()
    assert abs((host(ex) * D).sum() - want) <= 1e-5 * scale
    dw = rng.normal(size=50)
    f = lambda t: (orc.norm(host(x), host(w) + t * dw, host(b) + t * dw, 1e-5, kind)[0] * E).sum()
    assert abs(((host(gw) + host(gb)) * dw).sum() - (f(0.5) - f(-0.5))) <= 1e-5 * (np.abs(host(gw)) + np.abs(host(gb))).sum()


def test_bwd_nonfinite():
    """A NaN in E reaches its row of EX and its column of the sums, and nothing else."""
    x, w, _, rng = inputs(40, 300, torch.float32, torch.float32, 9)
    e = matrix(rng.normal(size=(40, 300)), torch.float32)
    mean, rstd = saved(x, "layer")
    clean = binding.halo_layer_norm_bwd(e, x, mean, rstd, w)
    e[7, 11] = float("nan")
    got = binding.halo_layer_norm_bwd(e, x, mean, rstd, w)
    rows, cols = [r for r in range(40) if r != 7], [c for c in range(300) if c != 11]
    assert torch.isnan(got[0][7]).all() and torch.equal(got[0][rows], clean[0][rows])
    for k in (1, 2):
        assert torch.isnan(got[k][11]) and torch.equal(got[k][cols], clean[k][cols])


def test_refusals():
    x = torch.zeros(4, 16, device=DEV)
    v = torch.zeros(16, device=DEV)
    for bad in (lambda: binding.halo_layer_norm_fwd(x, v[:15]), lambda: binding.halo_layer_norm_fwd(x, v, v.bfloat16()),
                lambda: binding.halo_layer_norm_fwd(x.t()), lambda: binding.halo_layer_norm_fwd(x, v, Y=x.bfloat16()),
                lambda: binding.halo_layer_norm_fwd(x, v, mean=v), lambda: binding.halo_layer_norm_bwd(x, x[:3], v[:4], v[:4], v),
                lambda: binding.halo_layer_norm_bwd(x, x, v[:4], v, v), lambda: binding.halo_layer_norm_bwd(x, x, v[:4], v[:4], v, GW=v[:4])):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(TypeError):
        binding.halo_layer_norm_fwd(x.half())
    with pytest.raises(ValueError):
        binding.halo_layer_norm_fwd(x, kind="batch")
    with pytest.raises(ValueError):
        binding.halo_layer_norm_fwd(x.cpu())
    with pytest.raises(binding.HaloError):
        binding.halo_layer_norm_bwd(x, x, None, v[:4], v)
    with pytest.raises(binding.HaloError):
        binding.halo_layer_norm_fwd(torch.zeros(1, 32776, device=DEV))
