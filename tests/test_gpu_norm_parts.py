"""halo_layer_norm_bwd with more rows than one launch takes: the sums of the columns are written in parts of the rows and joined by a second
launch.  Both kinds, with and without weight, base and each of the results, on both sides of every width that has a kernel of its own."""
import ctypes

import pytest
import torch

from paper_2501_02625_amd import binding
from tests.around_util import DTYPES, matrix, target
from tests.gpu_util import DEV
from tests.test_gpu_norm import KINDS, check_bwd, inputs, saved

pytestmark = pytest.mark.gpu


def case(rows, cols, dtype, wdtype, kind, seed, weight=True, base=True):
    x, w, _, rng = inputs(rows, cols, dtype, wdtype, seed)
    e = matrix(rng.normal(size=(rows, cols)), dtype, extra=1)
    b = matrix(rng.normal(size=(rows, cols)), dtype) if base else None
    return (e, x) + saved(x, kind) + (w if weight else None, b)


# columns: narrow ones share a workgroup's lanes, 128 lanes in teams of four up to 1024, then 256, 512 and 1024 lanes a row, four groups of 512
# lanes in bf16; beyond 8192 (fp32) and 16384 (bf16) the sums are in a launch of their own, with ragged ends too
@pytest.mark.parametrize("kind,weight", [("rms", True), ("rms", False), ("layer", False)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 40, 65, 200, 500, 1003, 2048, 4099, 8200, 16385, 32767])
def test_kinds_and_weights(cols, dtype, kind, weight):
    rows = 513 + cols % 200
    e, x, mean, rstd, w, base = case(rows, cols, dtype, DTYPES[cols % 2], kind, cols, weight, base=cols % 3 > 0)
    out, untouched = target(rows, cols, dtype)
    ex, gw, gb = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind=kind, base=base, EX=out)
    assert untouched()
    check_bwd(e, x, mean, rstd, w, base, kind, ex, gw, gb, "%s %d x %d" % (kind, rows, cols))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [40, 1003, 4096, 9000, 20000])
def test_each_output_alone(cols, dtype, kind):
    """The same numbers, whichever results are wanted, on a workspace of anything; E_X in the place of E, of base and of X."""
    rows = 700
    e, x, mean, rstd, w, base = case(rows, cols, dtype, dtype, kind, 6)
    whole = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind=kind, base=base)
    check_bwd(e, x, mean, rstd, w, base, kind, *whole, "%d x %d" % (rows, cols))
    ws = torch.full((1 << 27,), 255, dtype=torch.uint8, device=DEV)
    for want in range(1, 8):
        names = dict(want_ex=bool(want & 1), want_gw=bool(want & 2), want_gb=bool(want & 4))
        ws.fill_(255)
        got = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind=kind, base=base, workspace=ws, **names)
        for k in range(3):
            assert (got[k] is None) == (not want >> k & 1)
            assert got[k] is None or torch.equal(got[k], whole[k]), (want, k)
    for place in range(3):
        e2, b2, x2 = (matrix(t.double().cpu().numpy(), dtype) for t in (e, base, x))
        got = binding.halo_layer_norm_bwd(e2, x2, mean, rstd, w, kind=kind, base=b2, EX=(e2, b2, x2)[place], workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(got, whole)), place


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(3, 40), (300, 1003), (512, 8192), (513, 65), (700, 1003), (2000, 4096), (600, 8192), (1031, 9000), (513, 16384),
                                       (650, 20001)])
def test_workspace_is_as_large_as_asked(rows, cols, dtype):
    """Exactly the bytes that the query names: the results are the same, and what lies behind is not written."""
    e, x, mean, rstd, w, base = case(rows, cols, dtype, torch.float32, "layer", 7)
    whole = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base)
    d = binding.NormDesc(rows, cols, binding.HALO_NORM_KINDS["layer"], binding.HALO_F32 if dtype == torch.float32 else binding.HALO_BF16,
                         binding.HALO_F32, 0, 1e-5)
    need = binding.load_library().halo_layer_norm_bwd_workspace_bytes(ctypes.byref(d))
    buffer = torch.full((need + 65536,), 171, dtype=torch.uint8, device=DEV)
    got = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base, workspace=buffer[:need])
    assert all(torch.equal(a, b) for a, b in zip(got, whole))
    assert (buffer[need:] == 171).all()
    with pytest.raises(binding.HaloError) as refused:
        binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base, workspace=buffer[:need - 1])
    assert refused.value.status == binding.HALO_EWORKSPACE


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [65, 1003, 9000, 20001])
def test_nonfinite(cols, dtype, kind):
    """A NaN in E reaches its row of E_X and its columns of the sums, and nothing else; so does an infinity in X, but for G_B.  (With the saved
    statistics finite, an infinite xh makes the row's mean of d xh infinite, and E_X = rstd (d - mean - xh mean(d xh)) with it.)"""
    rows = 600
    e, x, mean, rstd, w, _ = case(rows, cols, dtype, torch.float32, kind, 9)
    clean = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind=kind)
    e[rows - 1, cols - 1], x[299, 11] = float("nan"), float("inf")
    ex, gw, gb = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind=kind)
    hit = torch.zeros(rows, dtype=torch.bool, device=DEV)
    hit[[299, rows - 1]] = True
    assert not torch.isfinite(ex[hit]).any() and torch.equal(ex[~hit], clean[0][~hit])
    columns = torch.arange(cols, device=DEV)
    for got, was, bad in ((gw, clean[1], (columns == cols - 1) | (columns == 11)), (gb, clean[2], columns == cols - 1)):
        assert not torch.isfinite(got[bad]).any() and torch.equal(got[~bad], was[~bad])


def test_few_rows_in_the_place_of_x():
    """E_X in the place of X where the sums of few rows are read beside it."""
    for cols in (40, 1003, 9000):
        e, x, mean, rstd, w, base = case(100, cols, torch.bfloat16, torch.float32, "layer", 10)
        whole = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base)
        got = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base, EX=x)
        assert got[0].data_ptr() == x.data_ptr() and all(torch.equal(a, b) for a, b in zip(got, whole))


@pytest.mark.parametrize("rows", [432, 433])
@pytest.mark.parametrize("cols", [4097, 8192])
def test_fp32_rows_of_16_to_32_kb(cols, rows):
    """Both sides of the number of rows from which on they take two launches."""
    e, x, mean, rstd, w, base = case(rows, cols, torch.float32, torch.float32, "layer", 11)
    ex, gw, gb = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base)
    check_bwd(e, x, mean, rstd, w, base, "layer", ex, gw, gb, "%d x %d" % (rows, cols))


def test_no_columns():
    """Results as empty as the matrix; statistics are refused (tests/test_norm_without_columns.py)."""
    x, v, w = torch.empty(5, 0, device=DEV), torch.ones(5, device=DEV), torch.empty(0, device=DEV)
    y, mean, rstd = binding.halo_layer_norm_fwd(x, w, w, want_stats=False)
    assert y.shape == (5, 0) and mean is None and rstd is None
    assert [t.shape for t in binding.halo_layer_norm_bwd(x, x, v, v, w)] == [(5, 0), (0,), (0,)]
    with pytest.raises(AssertionError):
        binding.halo_layer_norm_fwd(x)
