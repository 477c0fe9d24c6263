"""CPU checks of halo_dropout and halo_adapters_*: bad arguments are refused on the host before anything is launched."""
import ctypes
import os

import pytest
import torch

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


A, B, C = at(0x1000), at(0x20000), at(0x30000)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(dt=2), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL),
    (dict(p=-0.001), EINVAL), (dict(p=1.001), EINVAL), (dict(p=float("nan")), EINVAL), (dict(p=float("inf")), EINVAL),
    (dict(rows=(1 << 22) + 1), EUNSUPPORTED), (dict(ld=56), ESHAPE), (dict(ld_out=56), ESHAPE), (dict(res=B, ld_res=56), ESHAPE),
    (dict(out=A, ld_out=72), ESHAPE), (dict(res=C, ld_res=72), ESHAPE), (dict(x=at(0x1008)), EALIGN), (dict(out=at(0x30002)), EALIGN),
    (dict(res=at(0x20004), ld_res=64), EALIGN), (dict(ld=68), EALIGN), (dict(ld_out=65), EALIGN), (dict(res=B, ld_res=66), EALIGN),
    (dict(rows=0), OK), (dict(cols=0), OK),
])
def test_dropout(lib, change, status):
    a = dict(dict(x=A, dt=0, rows=16, cols=64, ld=64, res=None, ld_res=0, p=0.1, out=C, ld_out=64), **change)
    assert lib.halo_dropout(a["x"], a["dt"], a["rows"], a["cols"], a["ld"], a["res"], a["ld_res"], a["p"], 1, 2, a["out"], a["ld_out"],
                            None) == status


def desc(**change):
    a = dict(dict(b=16, m=64, n=128, slots=4, max_rank=16, out_dt=0, reserved=0, p=0.0), **change)
    return binding.AdaptersDesc(a["b"], a["m"], a["n"], a["slots"], a["max_rank"], a["out_dt"], a["reserved"], a["p"], 1, 2)


DESC_CHANGES = [
    (dict(b=-1), EINVAL), (dict(m=-8), EINVAL), (dict(n=-8), EINVAL), (dict(out_dt=2), EINVAL), (dict(reserved=1), EINVAL),
    (dict(p=-1.0), EINVAL), (dict(p=1.5), EINVAL), (dict(p=float("nan")), EINVAL), (dict(m=60), ESHAPE), (dict(n=129), ESHAPE),
    (dict(slots=0), ESHAPE), (dict(slots=-1), ESHAPE), (dict(max_rank=0), ESHAPE), (dict(max_rank=12), ESHAPE),
    (dict(max_rank=136), EUNSUPPORTED), (dict(slots=65536), EUNSUPPORTED), (dict(b=(1 << 22) + 1), EUNSUPPORTED),
    (dict(m=(1 << 22) + 8), EUNSUPPORTED),
]


def fwd(lib, d, **change):
    ld_y = 128
    a = dict(dict(X=A, ld_x=64, U=A, V=A, ranks=None, scale=None, of=A, base=None, ld_base=0, Y=C, ld_y=ld_y, T=B, ws=at(0x400000),
                  ws_bytes=1 << 40), **change)
    return lib.halo_adapters_fwd(ctypes.byref(d) if d else None, a["X"], a["ld_x"], a["U"], a["V"], a["ranks"], a["scale"], a["of"], a["base"],
                                 a["ld_base"], a["Y"], a["ld_y"], a["T"], a["ws"], a["ws_bytes"], None)


def bwd(lib, d, **change):
    a = dict(dict(E=A, ld_e=128, X=A, ld_x=64, T=A, U=A, V=A, ranks=None, scale=None, of=A, base=None, ld_base=0, EX=C, ld_ex=64, GU=B,
                  GV=at(0x50000), ws=at(0x400000), ws_bytes=1 << 40), **change)
    return lib.halo_adapters_bwd(ctypes.byref(d) if d else None, a["E"], a["ld_e"], a["X"], a["ld_x"], a["T"], a["U"], a["V"], a["ranks"],
                                 a["scale"], a["of"], a["base"], a["ld_base"], a["EX"], a["ld_ex"], a["GU"], a["GV"], a["ws"],
                                 a["ws_bytes"], None)


@pytest.mark.parametrize("change,status", DESC_CHANGES)
def test_descriptor(lib, change, status):
    d = desc(**change)
    assert fwd(lib, d) == status and bwd(lib, d) == status
    assert lib.halo_adapters_fwd_workspace_bytes(ctypes.byref(d)) == 0 and lib.halo_adapters_bwd_workspace_bytes(ctypes.byref(d)) == 0


def test_no_descriptor(lib):
    assert fwd(lib, None) == EINVAL and bwd(lib, None) == EINVAL
    assert lib.halo_adapters_fwd_workspace_bytes(None) == 0 and lib.halo_adapters_bwd_workspace_bytes(None) == 0


@pytest.mark.parametrize("change,status", [
    (dict(X=None), EINVAL), (dict(U=None), EINVAL), (dict(V=None), EINVAL), (dict(of=None), EINVAL), (dict(Y=None), EINVAL),
    (dict(T=None), EINVAL), (dict(ld_x=56), ESHAPE), (dict(ld_y=120), ESHAPE), (dict(base=B, ld_base=120), ESHAPE),
    (dict(base=C, ld_base=136), ESHAPE), (dict(ld_x=68), EALIGN), (dict(ld_y=132), EALIGN), (dict(base=B, ld_base=129), EALIGN),
    (dict(X=at(0x1008)), EALIGN), (dict(U=at(0x1002)), EALIGN), (dict(V=at(0x1002)), EALIGN), (dict(Y=at(0x30008)), EALIGN),
    (dict(T=at(0x20004)), EALIGN), (dict(base=at(0x20008), ld_base=128), EALIGN), (dict(of=at(0x1002)), EALIGN),
    (dict(ranks=at(0x1001)), EALIGN), (dict(scale=at(0x1002)), EALIGN),
])
def test_forward(lib, change, status):
    assert fwd(lib, desc(), **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(E=None), EINVAL), (dict(of=None), EINVAL), (dict(EX=None, GU=None, GV=None), EINVAL), (dict(U=None), EINVAL), (dict(V=None), EINVAL),
    (dict(X=None), EINVAL), (dict(T=None), EINVAL), (dict(ld_e=120), ESHAPE), (dict(ld_x=56), ESHAPE), (dict(ld_ex=56), ESHAPE),
    (dict(base=B, ld_base=56), ESHAPE), (dict(base=C, ld_base=72), ESHAPE), (dict(ld_e=132), EALIGN), (dict(ld_x=68), EALIGN),
    (dict(ld_ex=68), EALIGN), (dict(base=B, ld_base=68), EALIGN), (dict(E=at(0x1008)), EALIGN), (dict(GU=at(0x20004)), EALIGN),
    (dict(GV=at(0x20004)), EALIGN), (dict(EX=at(0x20004)), EALIGN), (dict(of=at(0x1002)), EALIGN),
])
def test_backward(lib, change, status):
    assert bwd(lib, desc(), **change) == status


def test_workspace(lib):
    """Where a pass needs a workspace, it is refused without one, with a byte too little, and at an address off 16 bytes."""
    for d, call, size in ((desc(), fwd, lib.halo_adapters_fwd_workspace_bytes), (desc(b=1), fwd, lib.halo_adapters_fwd_workspace_bytes),
                          (desc(b=2048, m=4096), fwd, lib.halo_adapters_fwd_workspace_bytes), (desc(), bwd, lib.halo_adapters_bwd_workspace_bytes),
                          (desc(b=2048, m=4096, out_dt=1), bwd, lib.halo_adapters_bwd_workspace_bytes)):
        need = size(ctypes.byref(d))
        lds = dict(ld_x=d.m, ld_ex=d.m) if call is bwd else dict(ld_x=d.m)
        if need:
            assert call(lib, d, ws=None, ws_bytes=0, **lds) == EWORKSPACE
            assert call(lib, d, ws_bytes=need - 1, **lds) == EWORKSPACE
            assert call(lib, d, ws=at(0x400008), **lds) == EALIGN
        else:
            assert call is fwd


def test_nothing_to_do(lib):
    for change in (dict(b=0), dict(m=0), dict(n=0)):
        assert fwd(lib, desc(**change), X=None, U=None, V=None, of=None, Y=None, T=None) == OK
    for change in (dict(m=0), dict(n=0)):
        assert bwd(lib, desc(**change), E=None, X=None, T=None, U=None, V=None, of=None) == OK


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.halo_dropout(x, 0.1, 1, 2)
    with pytest.raises(ValueError):
        binding.halo_adapters_fwd(x, x, x, x)
