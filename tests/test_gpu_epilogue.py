"""halo_gemm_i8_epilogue, halo_linear_fwd_epilogue and halo_activation_bwd against the formulas in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import around_oracle as orc
from paper_2501_02625_amd import binding
from tests.around_util import DTYPES, HALF, SLOPE, U, act_bound, column_terms, host, matrix, target, within
from tests.gpu_util import DEV, to_dev

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def operands(M, N, K, seed):
    rng = np.random.default_rng(seed)
    A, B = (rng.integers(-127, 128, size=(n, K)).astype(np.int8) for n in (M, N))
    rs = (0.5 + rng.random(M)).astype(np.float32)
    cs = ((0.5 + rng.random(N)) / (5400 * max(K, 1) ** 0.5)).astype(np.float32) * 2
    return A, B, rs, cs, rng


def check(A, B, rs, cs, bias, act, res, C, Z, dtype, what):
    y, z = orc.product(A, B, rs, cs, bias, act, res)
    plain = np.abs(z if bias is None else z - bias)
    off_z = 4 * U * plain + U * np.abs(z)
    if Z is not None:
        within(Z, z, off_z + HALF[dtype] * np.abs(z) * (1 + 1e-6), what + " Z")
    a = orc.act(z, act)
    # act's slope is at most 1.13
    bound = 1.2 * off_z + act_bound(z, a, act, dtype) + U * np.abs(y) + HALF[dtype] * (np.abs(y) + 1e-6)
    within(C, y, bound, what + " C")


# every kernel: 16 rows or fewer and 32 rows in tiles of 16, 32 and 64 columns, 64 x 64, 128 x 128, 256 x 128, 256 x 256, and sizes that
# end inside a tile in rows, columns and K
SHAPES = [(1, 16, 16), (1, 1000, 4096), (1, 4096, 4096), (3, 8192, 512), (16, 14336, 256), (17, 1024, 1008), (32, 4096, 1024), (32, 16384, 128),
          (64, 2048, 2064), (512, 2048, 512), (1000, 1003, 1008), (2048, 2048, 256), (1024, 4096, 4096), (4096, 4096, 400), (2999, 4093, 144),
          (4100, 8200, 128), (33, 1, 64), (300, 7, 96), (30, 8192, 128)]
# tiles of 256 x 192, alone and behind tiles of 256 x 256; rows that end inside one
TWO_WIDTHS = [(2199, 5312, 1024, torch.bfloat16), (4531, 5520, 256, torch.bfloat16), (1411, 7760, 2048, torch.float32),
              (4231, 6688, 1024, torch.float32)]


@pytest.mark.parametrize("M,N,K,dtype", [s + (d,) for s in SHAPES for d in DTYPES] + TWO_WIDTHS)
def test_product(M, N, K, dtype):
    A, B, rs, cs, rng = operands(M, N, K, M + N + K)
    act = ACTS[(M + N + K) % 5]
    bias = torch.tensor(0.3 * rng.normal(size=N)).to(DTYPES[M % 2]).to(DEV)
    res = matrix(rng.normal(size=(M, N)), dtype, extra=N % 2)
    out, untouched = target(M, N, dtype)
    zout, z_untouched = target(M, N, dtype, extra=2)
    C, Z = binding.halo_gemm_i8_epilogue(to_dev(A), to_dev(B), row_scale=to_dev(rs), col_scale=to_dev(cs), bias=bias, activation=act,
                                         residual=res, out=out, Z=zout)
    assert untouched() and z_untouched()
    check(A, B, rs, cs, host(bias), act, host(res), C, Z, dtype, "%s %d x %d x %d" % (act, M, N, K))


@pytest.mark.parametrize("M,N,K", [(5, 520, 64), (100, 1003, 144), (1030, 3000, 96)])
@pytest.mark.parametrize("act", ACTS)
def test_parts(act, M, N, K):
    """Each part of the epilogue there or not."""
    A, B, rs, cs, rng = operands(M, N, K, 1)
    bias = torch.tensor(0.3 * rng.normal(size=N), dtype=torch.float32, device=DEV)
    res = matrix(rng.normal(size=(M, N)), torch.float32)
    for with_bias in (False, True):
        for with_res in (False, True):
            for scales in (False, True):
                r, c = (rs, cs) if scales else (None, None)
                small = A // 32 if not scales else A
                C, Z = binding.halo_gemm_i8_epilogue(to_dev(small), to_dev(B if scales else B // 64), row_scale=None if r is None else to_dev(r),
                                                     col_scale=None if c is None else to_dev(c), bias=bias if with_bias else None,
                                                     activation=act, residual=res if with_res else None, want_z=with_bias)
                assert (Z is None) == (not with_bias)
                check(small, B if scales else B // 64, r, c, host(bias) if with_bias else None, act, host(res) if with_res else None, C, Z,
                      torch.float32, act)


@pytest.mark.parametrize("config", list(binding.HALO_GEMM_CONFIGS.values()))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N", [(256, 256), (300, 700), (129, 1001), (1, 17), (515, 130)])
def test_every_tile(M, N, dtype, config):
    K = 384
    A, B, rs, cs, rng = operands(M, N, K, 2)
    a, b, r, c = (to_dev(v) for v in (A, B, rs, cs))
    res, bias = matrix(rng.normal(size=(M, N)), dtype), torch.tensor(rng.normal(size=N), dtype=torch.bfloat16, device=DEV)
    out, untouched = target(M, N, dtype)
    z, z_untouched = target(M, N, dtype)
    g = binding.gemm_desc(a, b, trans_b=True, row_scale=r, col_scale=c, out=out, config=config)
    e = binding.Epilogue(bias.data_ptr(), 0, 4, res.data_ptr(), res.stride(0), z.data_ptr(), z.stride(0))
    st = binding.load_library().halo_gemm_i8_epilogue(ctypes.byref(g), ctypes.byref(e), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert st == binding.HALO_OK and untouched() and z_untouched()
    check(A, B, rs, cs, host(bias), "silu", host(res), out, z, dtype, "config %d" % config)


@pytest.mark.parametrize("M,N,K", [(7, 300, 64), (700, 1003, 128), (1024, 4096, 256)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_residual_in_place(dtype, M, N, K):
    A, B, rs, cs, rng = operands(M, N, K, 3)
    res = rng.normal(size=(M, N))
    args = dict(row_scale=to_dev(rs), col_scale=to_dev(cs), activation="gelu")
    want, _ = binding.halo_gemm_i8_epilogue(to_dev(A), to_dev(B), residual=matrix(res, dtype), out_dtype=dtype, **args)
    stream = matrix(res, dtype)
    got, _ = binding.halo_gemm_i8_epilogue(to_dev(A), to_dev(B), residual=stream, out=stream, **args)
    assert got is stream and torch.equal(got, want)


@pytest.mark.parametrize("M,N", [(3, 5), (40, 300), (2000, 2000)])
def test_no_activation_is_the_scaled_product(M, N):
    """Without bias, activation and residual: halo_gemm_i8, bit for bit."""
    A, B, rs, cs, _ = operands(M, N, 256, 4)
    a, b, r, c = (to_dev(v) for v in (A, B, rs, cs))
    for dtype in DTYPES:
        want, _ = binding.halo_gemm_i8(a, b, trans_b=True, row_scale=r, col_scale=c, out_dtype=dtype)
        C, Z = binding.halo_gemm_i8_epilogue(a, b, row_scale=r, col_scale=c, out_dtype=dtype, want_z=True)
        assert torch.equal(C, want) and torch.equal(Z, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_inner_dimension(dtype):
    bias, res = torch.arange(20.0, device=DEV) - 10, matrix(np.ones((5, 20)), dtype)
    a, b = torch.empty(5, 0, dtype=torch.int8, device=DEV), torch.empty(20, 0, dtype=torch.int8, device=DEV)
    C, Z = binding.halo_gemm_i8_epilogue(a, b, bias=bias, activation="relu", residual=res, out_dtype=dtype, want_z=True)
    assert torch.equal(C.float(), torch.relu(bias).expand(5, 20) + 1) and torch.equal(Z.float(), bias.expand(5, 20))


def test_nothing():
    a, b = torch.empty(0, 32, dtype=torch.int8, device=DEV), torch.zeros(20, 32, dtype=torch.int8, device=DEV)
    assert binding.halo_gemm_i8_epilogue(a, b)[0].shape == (0, 20) and binding.halo_gemm_i8_epilogue(b, a)[0].shape == (20, 0)


def test_large_values_and_nonfinite():
    """Each activation at large and infinite arguments, and what lies next to them untouched: bias reaches its column, residual its element."""
    for act in ACTS:
        for M, N in ((4, 64), (300, 600)):
            a, b = torch.zeros(M, 32, dtype=torch.int8, device=DEV), torch.zeros(N, 32, dtype=torch.int8, device=DEV)
            bias = torch.zeros(N, device=DEV)
            values = [1e30, -1e30, 100.0, -100.0, float("inf"), float("nan"), 20.0, -20.0]
            bias[3:11] = torch.tensor(values)
            res = torch.ones(M, N, device=DEV)
            res[1, 1], res[2, 2] = float("inf"), float("nan")
            C, _ = binding.halo_gemm_i8_epilogue(a, b, bias=bias, activation=act, residual=res, out_dtype=torch.float32)
            y = orc.act(np.array(values[:4] + values[6:]), act) + 1
            got = host(C[0, [3, 4, 5, 6, 9, 10]])
            # act none keeps -1e30 and -100; the others tend to 0 there
            assert np.allclose(got, y, rtol=1e-6, atol=1e-6), (act, got, y)
            assert torch.isinf(C[0, 7]) and torch.isnan(C[0, 8])
            assert torch.isinf(C[1, 1]) and torch.isnan(C[2, 2])
            rest = torch.ones(M, N, dtype=torch.bool, device=DEV)
            rest[:, 3:11] = False
            rest[1, 1] = rest[2, 2] = False
            assert (C[rest] == 1).all()


@pytest.mark.parametrize("mode", [binding.HALO_SCALE_PER_ROW, binding.HALO_SCALE_PER_TENSOR])
@pytest.mark.parametrize("level", [0, 1, 2])
@pytest.mark.parametrize("dtype", DTYPES)
def test_layer(dtype, level, mode):
    """The codes and scales are those of halo_linear_fwd; Y is the epilogue of their product."""
    b, m, n = 48, 256, 80
    g = torch.Generator(device=DEV).manual_seed(5)
    X, W = (torch.randn(*s, generator=g, device=DEV).bfloat16() for s in ((b, m), (n, m)))
    bias, res = torch.randn(n, generator=g, device=DEV), torch.randn(b, n, generator=g, device=DEV).to(dtype)
    desc = binding.make_desc(b, m, n, level, dtype, scale_mode=mode)
    Y0, s0 = binding.halo_linear_fwd(desc, X, W)
    Y, s, Z = binding.halo_linear_fwd_epilogue(desc, X, W, bias=bias, activation="gelu", residual=res, want_z=True)
    assert all(torch.equal(getattr(s, k), getattr(s0, k)) for k in ("Xq", "s_x", "Wq", "s_w"))
    check(s.Xq.cpu().numpy(), s.Wq.cpu().numpy(), s.s_x.cpu().numpy(), s.s_w.cpu().numpy(), host(bias), "gelu", host(res), Y, Z, dtype, "layer")
    again, same, none = binding.halo_linear_fwd_epilogue(desc, X, None, state=s, Y=res, bias=bias, activation="gelu", residual=res)
    assert same is s and none is None and again is res and torch.equal(again, Y)
    plain, _, _ = binding.halo_linear_fwd_epilogue(desc, X, W)
    assert torch.equal(plain, Y0)


def test_refusals():
    a, b = torch.zeros(4, 32, dtype=torch.int8, device=DEV), torch.zeros(8, 32, dtype=torch.int8, device=DEV)
    v, m = torch.zeros(8, device=DEV), torch.zeros(4, 8, device=DEV)
    for bad in (dict(bias=v[:7]), dict(bias=v.double()), dict(residual=m.bfloat16()), dict(residual=m[:3]), dict(Z=m.bfloat16()), dict(row_scale=v),
                dict(out=torch.zeros(4, 9, device=DEV))):
        with pytest.raises((AssertionError, TypeError)):
            binding.halo_gemm_i8_epilogue(a, b, **bad)
    with pytest.raises(ValueError):
        binding.halo_gemm_i8_epilogue(a, b, activation="tanh")
    with pytest.raises(ValueError):
        binding.halo_gemm_i8_epilogue(a, b.cpu())
    with pytest.raises(AssertionError):
        binding.halo_gemm_i8_epilogue(a, b[:, :16])
    with pytest.raises(binding.HaloError):
        binding.halo_gemm_i8_epilogue(a, b, residual=m, Z=m)
    with pytest.raises(binding.HaloError):
        binding.halo_gemm_i8_epilogue(a[:, :20].contiguous(), b[:, :20].contiguous())


# ------------------------------------------------------------------------------------------------ the gradient
def check_grad(e, z, act, ez, gb, what):
    E, Z = host(e), host(z) if z is not None else np.zeros(e.shape)
    d = E * orc.slope(Z, act)
    exact = act in ("none", "relu")
    off = 0.0 if exact else SLOPE * np.abs(E)
    if ez is not None:
        within(ez, d, off + HALF[e.dtype] * np.abs(d) * (1 + 1e-5), what + " EZ")
    if gb is not None:
        within(gb, d.sum(axis=0), (off + np.zeros(E.shape)).sum(axis=0) + column_terms(len(E)) * U * np.abs(d).sum(axis=0), what + " GB")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (16, 64), (129, 513), (1000, 1003), (2, 14336), (5000, 40), (300, 4104), (70000, 9)])
def test_activation_bwd(rows, cols, dtype, act):
    rng = np.random.default_rng(rows + cols)
    e, z = matrix(rng.normal(size=(rows, cols)), dtype, extra=1), matrix(3 * rng.normal(size=(rows, cols)), dtype)
    out, untouched = target(rows, cols, dtype)
    ez, gb = binding.halo_activation_bwd(e, None if act == "none" else z, act, EZ=out)
    assert untouched()
    check_grad(e, z, act, ez, gb, "%s %d x %d" % (act, rows, cols))


def test_activation_bwd_each_output_alone():
    rng = np.random.default_rng(6)
    for dtype in DTYPES:
        e, z = (matrix(rng.normal(size=(700, 1003)), dtype) for _ in range(2))
        ez, gb = binding.halo_activation_bwd(e, z, "silu")
        assert torch.equal(binding.halo_activation_bwd(e, z, "silu", want_gb=False)[0], ez)
        ws = torch.full((1 << 22,), 255, dtype=torch.uint8, device=DEV)
        assert torch.equal(binding.halo_activation_bwd(e, z, "silu", want_ez=False, workspace=ws)[1], gb)
        for place in (0, 1):
            e2, z2 = (matrix(t.float().cpu().numpy(), dtype) for t in (e, z))
            got, gb2 = binding.halo_activation_bwd(e2, z2, "silu", EZ=(e2, z2)[place])
            assert torch.equal(got, ez) and torch.equal(gb2, gb)


def test_activation_bwd_of_no_rows():
    e = torch.empty(0, 33, device=DEV)
    ez, gb = binding.halo_activation_bwd(e, e, "gelu", GB=torch.ones(33, device=DEV))
    assert ez.shape == (0, 33) and not gb.any()
    assert binding.halo_activation_bwd(torch.empty(5, 0, device=DEV), torch.empty(5, 0, device=DEV), "gelu")[0].shape == (5, 0)


@pytest.mark.parametrize("act", ACTS[1:])
def test_slopes_far_out(act):
    """Slopes are 0 and 1 at the ends, at infinities too; a NaN is its own element's and its column's."""
    z = torch.tensor([[1e30, -1e30, 200.0, -200.0, float("inf"), float("-inf"), float("nan"), 0.0, 15.0, -15.0]], device=DEV)
    ez, gb = binding.halo_activation_bwd(torch.full_like(z, 2.0), z, act)
    at_zero = {"relu": 0.0}.get(act, 1.0)
    want = torch.tensor([2.0, 0.0, 2.0, 0.0, 2.0, 0.0, float("nan"), at_zero, 2.0, 0.0], device=DEV)
    assert torch.allclose(ez[0], want, rtol=0, atol=2e-4 if act == "silu" else 1e-6, equal_nan=True) and torch.equal(torch.isnan(gb), torch.isnan(z[0]))


@pytest.mark.parametrize("act", ACTS)
def test_gradient_is_that_of_the_epilogue(act):
    """Differences of the oracle's forward pass, in 64 bits, along a direction of Z and of the bias."""
    rng = np.random.default_rng(7)
    z = matrix(rng.normal(size=(30, 17)) * 2, torch.float32)
    E, D, h = rng.normal(size=(30, 17)), rng.normal(size=17), 1e-5
    _, gb = binding.halo_activation_bwd(matrix(E, torch.float32), z, act)
    f = lambda t: (orc.act(host(z) + t * D, act) * E).sum()
    assert abs((host(gb) * D).sum() - (f(h) - f(-h)) / (2 * h)) <= 1e-5 * np.abs(E * D).sum()
