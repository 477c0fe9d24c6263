"""GPU: infinities and NaN among what halo_adapters_* take reach what the formulas say, and nothing else."""
import numpy as np
import pytest
import torch

from tests import gpu_util as gu
from tests.test_gpu_adapters import Case, runs

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
