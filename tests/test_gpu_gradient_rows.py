"""The gradients of the norm and of an epilogue on both sides of the numbers of rows from which on the sums of the columns are joined in a
second launch, for every width that has kernels of its own."""
import numpy as np
import pytest
import torch

from paper_2501_02625_amd import binding
from tests.around_util import DTYPES, matrix, target
from tests.gpu_util import DEV
from tests.test_gpu_epilogue import check_grad
from tests.test_gpu_norm import check_bwd, inputs, saved

pytestmark = pytest.mark.gpu
WIDTHS = [40, 65, 200, 500, 1003, 2048, 4099, 8192, 9000, 16384]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm(cols, dtype):
    for rows in (127, 256, 257, 512, 513):
        x, w, _, rng = inputs(rows, cols, dtype, DTYPES[rows % 2], rows + cols)
        e, base = matrix(rng.normal(size=(rows, cols)), dtype, extra=1), matrix(rng.normal(size=(rows, cols)), dtype)
        mean, rstd = saved(x, "layer")
        out, untouched = target(rows, cols, dtype)
        ex, gw, gb = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, base=base, EX=out)
        assert untouched()
        check_bwd(e, x, mean, rstd, w, base, "layer", ex, gw, gb, "%d x %d" % (rows, cols))
        again = matrix(e.double().cpu().numpy(), dtype)
        got = binding.halo_layer_norm_bwd(again, x, mean, rstd, w, base=base, EX=again)
        assert all(torch.equal(a, b) for a, b in zip(got, (ex, gw, gb)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_activation(cols, dtype):
    for rows in (33, 128, 129, 261):
        rng = np.random.default_rng(rows + cols)
        e, z = matrix(rng.normal(size=(rows, cols)), dtype, extra=1), matrix(2 * rng.normal(size=(rows, cols)), dtype)
        out, untouched = target(rows, cols, dtype)
        ez, gb = binding.halo_activation_bwd(e, z, "gelu", EZ=out)
        assert untouched()
        check_grad(e, z, "gelu", ez, gb, "%d x %d" % (rows, cols))
        for place in (0, 1):
            e2, z2 = (matrix(t.double().cpu().numpy(), dtype) for t in (e, z))
            got, gb2 = binding.halo_activation_bwd(e2, z2, "gelu", EZ=(e2, z2)[place])
            assert torch.equal(got, ez) and torch.equal(gb2, gb)


@pytest.mark.parametrize("rows", [100, 700])
def test_nonfinite_columns_stay_columns(rows):
    x, w, _, rng = inputs(rows, 1003, torch.float32, torch.float32, 8)
    e = matrix(rng.normal(size=(rows, 1003)), torch.float32)
    mean, rstd = saved(x, "rms")
    clean = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind="rms")
    clean_gb = binding.halo_activation_bwd(e, x, "silu")[1]
    e[rows - 1, 1002], e[3, 64] = float("nan"), float("inf")
    got = binding.halo_layer_norm_bwd(e, x, mean, rstd, w, kind="rms")
    keep = torch.ones(1003, dtype=torch.bool, device=DEV)
    keep[[64, 1002]] = False
    for a, b in zip(got[1:] + (binding.halo_activation_bwd(e, x, "silu")[1],), clean[1:] + (clean_gb,)):
        assert torch.equal(a[keep], b[keep]) and not torch.isfinite(a[~keep]).any()
    rows_kept = [r for r in range(rows) if r not in (3, rows - 1)]
    assert torch.equal(got[0][rows_kept], clean[0][rows_kept])


@pytest.mark.parametrize("rows", [100, 700])
def test_captured(rows):
    """A graph of both gradients replayed with new inputs, among eager calls."""
    x, w, _, rng = inputs(rows, 1003, torch.bfloat16, torch.bfloat16, 9)
    e = matrix(rng.normal(size=(rows, 1003)), torch.bfloat16)
    mean, rstd = saved(x, "layer")

    def both():
        ez, gb = binding.halo_activation_bwd(e, x, "gelu_tanh")
        return (ez, gb) + tuple(binding.halo_layer_norm_bwd(ez, x, mean, rstd, w))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(3):
        e.copy_(torch.tensor(rng.normal(size=(rows, 1003))).to(DEV))
        want = both()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
