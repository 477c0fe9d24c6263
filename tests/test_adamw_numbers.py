"""halo_adamw with its step, rate and scale in device memory: refused where the call would write over them while its workgroups read them (CPU),
done where they lie next to what is written, or share a place with what is only read (GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2501_02625_amd import binding
from tests.test_around_abi import adamw, lib, tensor  # noqa: F401 (lib: a fixture)

# of tensor(0): where it lies, 1000 fp32 elements
PARAM, M, V, M_SCALE, V_SCALE, MASTER = (0x10000000 + k * 0x100000 for k in (0, 2, 3, 4, 5, 6))


@pytest.mark.parametrize("at", [PARAM, PARAM + 1000, M + 992, V, M_SCALE + 8, V_SCALE])
@pytest.mark.parametrize("name", ["step_ptr", "lr_ptr", "gs_ptr"])
def test_in_what_is_written(lib, name, at):  # noqa: F811
    assert adamw(lib, param_dt=1, **{name: at}) == binding.HALO_EINVAL


def test_across_a_border(lib):  # noqa: F811
    """Of the step's eight bytes the first four are a parameter's last element; the rate is a master copy's last; the scale a second tensor's."""
    assert adamw(lib, [tensor(0, size=999)], param_dt=1, step_ptr=PARAM + 3992) == binding.HALO_EINVAL
    assert adamw(lib, [tensor(0, master=MASTER)], param_dt=0, lr_ptr=MASTER + 3996) == binding.HALO_EINVAL
    assert adamw(lib, [tensor(0), tensor(1)], gs_ptr=0x20000000 + 64) == binding.HALO_EINVAL


@pytest.mark.gpu
def test_next_to_what_is_written():
    from tests.gpu_util import DEV

    def made():
        """param (500 elements), then the rate, the scale and, eight bytes on, the step; the rate is an element of the gradient too."""
        g = torch.Generator(device=DEV).manual_seed(1)
        buffer = torch.zeros(512, device=DEV)
        grad = torch.randn(500, generator=g, device=DEV)
        buffer[:500] = torch.randn(500, generator=g, device=DEV)
        grad[3] = 1e-2
        return buffer, grad, [torch.zeros(500, device=DEV)], [torch.zeros(500, device=DEV)]

    buffer, grad, m, v = made()
    buffer[501] = 0.5
    step = buffer[502:504].view(torch.int64)
    step.fill_(7)
    binding.halo_adamw([buffer[:500]], [grad], m, v, step=step, lr=grad[3:4], grad_scale=buffer[501:502])
    other, grad2, m2, v2 = made()
    binding.halo_adamw([other[:500]], [grad2], m2, v2, step=7, lr=float(np.float32(1e-2)), grad_scale=0.5)
    assert torch.equal(buffer[:500], other[:500]) and torch.equal(m[0], m2[0]) and torch.equal(v[0], v2[0])
    assert buffer[500] == 0 and buffer[501] == 0.5 and step.item() == 7
