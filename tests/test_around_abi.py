"""CPU checks of halo_gemm_i8_epilogue, halo_linear_fwd_epilogue, halo_activation_bwd, halo_layer_norm_* and halo_adamw: bad arguments are
refused on the host before anything is launched."""
import ctypes
import os

import pytest

from paper_2501_02625_amd import _build, binding

OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE, EUNSUPPORTED = (binding.HALO_OK, binding.HALO_EINVAL, binding.HALO_ESHAPE, binding.HALO_EALIGN,
                                                        binding.HALO_EWORKSPACE, binding.HALO_EUNSUPPORTED)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    return binding.load_library()


def at(v):
    return ctypes.c_void_p(v)


A, B, C, D = 0x1000, 0x200000, 0x400000, 0x600000


# ---- epilogue
EPILOGUE = [
    (dict(activation=5), EINVAL), (dict(activation=-1), EINVAL), (dict(bias=A, bias_dt=2), EINVAL), (dict(bias=A + 4), EALIGN),
    (dict(residual=A, ld_res=120), ESHAPE), (dict(residual=C, ld_res=136), ESHAPE), (dict(residual=A + 8, ld_res=128), EALIGN),
    (dict(residual=A, ld_res=129), EALIGN), (dict(Z=C, ld_z=128), EINVAL), (dict(Z=A, ld_z=120), ESHAPE), (dict(Z=A + 2, ld_z=128), EALIGN),
    (dict(Z=A, ld_z=130), EALIGN), (dict(Z=D, ld_z=128, residual=D, ld_res=128), EINVAL),
]


def epilogue(**change):
    a = dict(dict(bias=None, bias_dt=1, activation=2, residual=None, ld_res=0, Z=None, ld_z=0), **change)
    return binding.Epilogue(*a.values())


def product(lib, e, **change):
    a = dict(dict(A=A, lda=64, B=B, ldb=64, transB=1, M=32, N=128, K=64, rs=None, cs=None, C=C, c_dt=0, ldc=128, acc=None, ld_acc=0, config=-1),
             **change)
    g = binding.GemmDesc(*a.values())
    return lib.halo_gemm_i8_epilogue(ctypes.byref(g), None if e is None else ctypes.byref(e), None)


@pytest.mark.parametrize("change,status", EPILOGUE)
def test_epilogue(lib, change, status):
    assert product(lib, epilogue(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(C=None), EINVAL), (dict(C=None, acc=D, ld_acc=128), EINVAL), (dict(acc=D, ld_acc=128), EINVAL), (dict(transB=0, ldb=128), EUNSUPPORTED),
    (dict(K=60), ESHAPE), (dict(c_dt=3), EINVAL), (dict(M=-1), EINVAL), (dict(lda=48), ESHAPE), (dict(ldc=120), ESHAPE), (dict(C=C + 8), EALIGN),
    (dict(K=1 << 18, lda=1 << 18, ldb=1 << 18), ESHAPE), (dict(M=0), OK), (dict(N=0), OK), (dict(config=9), EINVAL),
])
def test_product(lib, change, status):
    assert product(lib, epilogue(), **change) == status


def test_no_epilogue(lib):
    assert product(lib, None) == EINVAL
    assert lib.halo_gemm_i8_epilogue(None, ctypes.byref(epilogue()), None) == EINVAL


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("change,status", EPILOGUE)
def test_layer(lib, change, status, mode):
    """Refused before the operands are quantised."""
    d = binding.LinearDesc(32, 64, 128, 1, 0, 0, 0, mode)
    e = epilogue(**change)
    st = lib.halo_linear_fwd_epilogue(ctypes.byref(d), at(A), at(B), at(C), at(0x10000), at(0x20000), at(0x30000), at(0x40000), ctypes.byref(e),
                                      at(0x800000), 1 << 40, None)
    assert st == status


# ---- activation's gradient
@pytest.mark.parametrize("change,status", [
    (dict(E=None), EINVAL), (dict(Z=None), EINVAL), (dict(EZ=None, GB=None), EINVAL), (dict(dt=2), EINVAL), (dict(act=5), EINVAL),
    (dict(act=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL), (dict(rows=(1 << 22) + 1), EUNSUPPORTED),
    (dict(cols=(1 << 22) + 8, ld_e=1 << 23, ld_z=1 << 23, ld_ez=1 << 23), EUNSUPPORTED), (dict(ld_e=56), ESHAPE), (dict(ld_z=56), ESHAPE),
    (dict(ld_ez=56), ESHAPE), (dict(EZ=A, ld_ez=72), ESHAPE), (dict(EZ=B, ld_ez=72), ESHAPE), (dict(E=A + 8), EALIGN), (dict(ld_z=65), EALIGN),
    (dict(EZ=C + 2), EALIGN), (dict(GB=D + 4), EALIGN), (dict(ws=None), EWORKSPACE), (dict(bytes=4), EWORKSPACE), (dict(ws=0x800004), EALIGN),
    (dict(cols=0), OK), (dict(rows=0, GB=None), OK),
])
def test_activation_bwd(lib, change, status):
    a = dict(dict(E=A, ld_e=64, Z=B, ld_z=64, dt=0, rows=16, cols=64, act=2, EZ=C, ld_ez=64, GB=D, ws=0x800000, bytes=1 << 40), **change)
    assert lib.halo_activation_bwd(a["E"], a["ld_e"], a["Z"], a["ld_z"], a["dt"], a["rows"], a["cols"], a["act"], a["EZ"], a["ld_ez"], a["GB"],
                                   a["ws"], a["bytes"], None) == status


def test_workspaces_of_nothing(lib):
    for rows, cols in ((0, 64), (16, 0), (-1, 64), (16, -1), ((1 << 22) + 1, 64)):
        assert lib.halo_activation_bwd_workspace_bytes(rows, cols) == 0
    assert lib.halo_activation_bwd_workspace_bytes(16, 64) > 0
    for change in (dict(rows=0), dict(cols=0), dict(rows=-1), dict(cols=32769), dict(dt=7), dict(reserved=1)):
        assert lib.halo_layer_norm_bwd_workspace_bytes(ctypes.byref(norm(**change))) == 0
    assert lib.halo_layer_norm_bwd_workspace_bytes(None) == 0


# ---- norm
def norm(**change):
    a = dict(dict(rows=16, cols=64, kind=0, dt=0, weight_dt=1, reserved=0, eps=1e-5), **change)
    return binding.NormDesc(*a.values())


def fwd(lib, d, **change):
    a = dict(dict(X=A, ld_x=64, w=B, b=None, Y=C, ld_y=64, mean=None, rstd=None), **change)
    return lib.halo_layer_norm_fwd(ctypes.byref(d) if d else None, *a.values(), None)


def bwd(lib, d, **change):
    a = dict(dict(E=A, ld_e=64, X=B, ld_x=64, mean=A, rstd=A, w=B, base=None, ld_base=0, EX=C, ld_ex=64, GW=D, GB=D + 4096, ws=0x800000,
                  bytes=1 << 40), **change)
    return lib.halo_layer_norm_bwd(ctypes.byref(d) if d else None, *a.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL), (dict(kind=2), EINVAL), (dict(dt=2), EINVAL), (dict(weight_dt=-1), EINVAL),
    (dict(reserved=1), EINVAL), (dict(eps=-1e-5), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL),
    (dict(eps=1e300), EINVAL), (dict(cols=32769), EUNSUPPORTED), (dict(rows=1 << 31), EUNSUPPORTED),
])
def test_norm_descriptor(lib, change, status):
    assert fwd(lib, norm(**change)) == status and bwd(lib, norm(**change)) == status


def test_no_norm(lib):
    assert fwd(lib, None) == EINVAL and bwd(lib, None) == EINVAL
    assert fwd(lib, norm(rows=0), X=None) == OK and fwd(lib, norm(cols=0), X=None) == OK and bwd(lib, norm(cols=0), E=None) == OK
    assert bwd(lib, norm(rows=0), E=None, GW=None, GB=None) == OK


@pytest.mark.parametrize("change,status", [
    (dict(X=None), EINVAL), (dict(Y=None), EINVAL), (dict(ld_x=56), ESHAPE), (dict(ld_y=56), ESHAPE), (dict(Y=A, ld_y=72), ESHAPE),
    (dict(X=A + 8), EALIGN), (dict(ld_y=65), EALIGN), (dict(w=B + 8), EALIGN), (dict(b=B + 4), EALIGN), (dict(mean=D + 2), EALIGN),
    (dict(rstd=D + 1), EALIGN),
])
def test_norm_fwd(lib, change, status):
    assert fwd(lib, norm(), **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(E=None), EINVAL), (dict(X=None), EINVAL), (dict(rstd=None), EINVAL), (dict(mean=None), EINVAL), (dict(EX=None, GW=None, GB=None), EINVAL),
    (dict(ld_e=56), ESHAPE), (dict(ld_x=56), ESHAPE), (dict(ld_ex=56), ESHAPE), (dict(base=D, ld_base=56), ESHAPE), (dict(EX=A, ld_ex=72), ESHAPE),
    (dict(base=C, ld_base=72), ESHAPE), (dict(E=A + 2), EALIGN), (dict(X=B + 8), EALIGN), (dict(EX=C + 4), EALIGN), (dict(base=D, ld_base=65), EALIGN),
    (dict(w=B + 2), EALIGN), (dict(GW=D + 4), EALIGN), (dict(GB=D + 8), EALIGN), (dict(ws=None), EWORKSPACE), (dict(bytes=16), EWORKSPACE),
    (dict(ws=0x800008), EALIGN),
])
def test_norm_bwd(lib, change, status):
    assert bwd(lib, norm(), **change) == status


# ---- AdamW
def adamw(lib, tensors=None, count=None, **change):
    a = dict(dict(param_dt=0, grad_dt=0, bits=8, reserved=0, step=1, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, wd=0.1, gs=1.0, seed=1, offset=2,
                  step_ptr=None, lr_ptr=None, gs_ptr=None), **change)
    d = binding.AdamwDesc(*a.values())
    tensors = [tensor(0)] if tensors is None else tensors
    arr = (binding.AdamwTensor * max(1, len(tensors)))(*tensors)
    return lib.halo_adamw(ctypes.byref(d), arr, len(tensors) if count is None else count, None)


def tensor(k, **change):
    base = 0x10000000 * (k + 1)
    a = dict(dict(size=1000, param=base, grad=base + 0x100000, m=base + 0x200000, v=base + 0x300000, master=None, m_scale=base + 0x400000,
                  v_scale=base + 0x500000), **change)
    return binding.AdamwTensor(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(param_dt=2), EINVAL), (dict(grad_dt=-1), EINVAL), (dict(bits=16), EINVAL), (dict(reserved=1), EINVAL), (dict(step=0), EINVAL),
    (dict(lr=-1.0), EINVAL), (dict(lr=float("nan")), EINVAL), (dict(lr=1e300), EINVAL), (dict(beta1=1.0), EINVAL), (dict(beta1=-0.1), EINVAL),
    (dict(beta2=1.0), EINVAL), (dict(beta2=1 - 1e-12), EINVAL), (dict(beta2=float("nan")), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(wd=-0.1), EINVAL), (dict(gs=float("inf")), EINVAL), (dict(gs=float("nan")), EINVAL), (dict(step_ptr=A + 4), EALIGN),
    (dict(lr_ptr=A + 2), EALIGN), (dict(gs_ptr=A + 1), EALIGN), (dict(count=-1), EINVAL), (dict(count=1025), EUNSUPPORTED), (dict(count=0), OK),
])
def test_adamw(lib, change, status):
    assert adamw(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(size=-1), EINVAL), (dict(param=None), EINVAL), (dict(grad=None), EINVAL), (dict(m=None), EINVAL), (dict(v=None), EINVAL),
    (dict(m_scale=None), EINVAL), (dict(v_scale=None), EINVAL), (dict(size=(1 << 34) + 1), EUNSUPPORTED), (dict(param=0x20000008), EALIGN),
    (dict(grad=0x20000002), EALIGN), (dict(m=0x20000004), EALIGN), (dict(v=0x20000008), EALIGN), (dict(master=0x20600004), EALIGN),
    (dict(m_scale=0x20400002), EALIGN), (dict(v_scale=0x20500001), EALIGN), (dict(m=0x20000000), EINVAL), (dict(m_scale=0x20300000), EINVAL),
    (dict(param=0x10000000), EINVAL), (dict(param=0x10000000 + 1984), EINVAL), (dict(v=0x10300000 + 992), EINVAL), (dict(master=0x20600000), EINVAL),
    (dict(grad=0x10000000), EINVAL), (dict(grad=0x20200000), EINVAL), (dict(m=0x10100000), EINVAL), (dict(param=0x10100000 + 1984), EINVAL),
])
def test_adamw_tensors(lib, change, status):
    """The second of two tensors: missing, misaligned, or overlapping the first or itself; one master for two."""
    assert adamw(lib, [tensor(0), tensor(1, **change)]) == status


def test_adamw_masters_of_fp32(lib):
    assert adamw(lib, [tensor(0, master=0x10600000)], param_dt=1) == EINVAL


def test_adamw_nothing_to_do(lib):
    assert adamw(lib, [tensor(0, size=0, param=None, grad=None), tensor(1, size=0)]) == OK
