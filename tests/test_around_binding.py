"""CPU tests of the binding of the operators around a layer's products: what it refuses before it calls the library.  In a process of their
own, on fake device tensors (no GPU is used)."""
import pytest

from tests.test_native_binding import run

CALLS = {
    "epilogue": "binding.halo_gemm_i8_epilogue(new(4, 32, dtype=i8), new(8, 32, dtype=i8), {0}=new(8, dtype=f32, device='{1}'))",
    "layer": "binding.halo_linear_fwd_epilogue(desc, new(16, 64), new(32, 64), {0}=new(32, dtype=f32, device='{1}'))",
    "activation": "binding.halo_activation_bwd(new(4, 32), new(4, 32, device='{1}'), 'gelu')",
    "norm": "binding.halo_layer_norm_fwd(new(4, 32), new(32, device='{1}'))",
    "norm gradient": "binding.halo_layer_norm_bwd(new(4, 32), new(4, 32), new(4, dtype=f32), new(4, dtype=f32), new(32, device='{1}'))",
    "adamw": "binding.halo_adamw([new(8)], [new(8, device='{1}')], [new(8, dtype=f32)], [new(8, dtype=f32)], step=1, lr=0.1)",
    "adamw's step": "binding.halo_adamw([new(8)], [new(8)], [new(8, dtype=f32)], [new(8, dtype=f32)], step=new(1, dtype=torch.int64, device='{1}'), lr=0.1)",
}


@pytest.mark.parametrize("device,what", [("cuda:1", "tensors are on the current device"), ("cpu", "libhalo takes device tensors only")])
def test_tensors_elsewhere(device, what):
    """On another device than the current one, whose stream the call would go to, or on the host."""
    body = """
def new(*shape, dtype=bf, device="cuda:0"):
    return torch.empty(shape, dtype=dtype, device=device)
with FakeTensorMode():
    for f in (%s):
        try:
            f()
            print("went through")
        except ValueError as e:
            print(e)
""" % ", ".join("lambda: " + c.format("bias", device) for c in CALLS.values())
    assert run(body).splitlines() == [what] * len(CALLS)


def test_names():
    out = run("""
with FakeTensorMode():
    x, v = new(4, 32), new(4, dtype=f32)
    for f in (lambda: binding.halo_gemm_i8_epilogue(new(4, 32, dtype=i8), new(8, 32, dtype=i8), activation="swish"),
              lambda: binding.halo_activation_bwd(x, x, "GELU"), lambda: binding.halo_layer_norm_fwd(x, kind="batch"),
              lambda: binding.halo_layer_norm_bwd(x, x, v, v, kind=0)):
        try:
            f()
            print("went through")
        except ValueError as e:
            print("refused")
""")
    assert out.split() == ["refused"] * 4


def test_rows_that_overlap():
    """Expanded matrices have rows 0 elements apart: refused, as any pitch below the row's length."""
    out = run("""
with FakeTensorMode():
    x, v = new(1, 32).expand(4, 32), new(4, dtype=f32)
    for f in (lambda: binding.halo_activation_bwd(x, x, "gelu"), lambda: binding.halo_layer_norm_fwd(x),
              lambda: binding.halo_layer_norm_bwd(x, new(4, 32), v, v),
              lambda: binding.halo_gemm_i8_epilogue(new(1, 32, dtype=i8).expand(4, 32), new(8, 32, dtype=i8))):
        try:
            f()
            print("went through")
        except binding.HaloError as e:
            print(e.status in (binding.HALO_ESHAPE, binding.HALO_EINVAL))
""")
    assert out.split() == ["True"] * 4
