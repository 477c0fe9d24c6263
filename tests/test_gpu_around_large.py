"""Offsets beyond 32 bits and pitches beyond what tiles take."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as orc
from paper_2501_02625_amd import binding
from tests.around_util import HALF, U, act_bound, column_terms, host, within
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_adamw_beyond_2_to_32_elements():
    """One tensor of 2^32 + 777 elements, bf16 with states in 8 bits: places at the start, about 2^31 and 2^32, and the end."""
    n = 2 ** 32 + 777
    g = torch.Generator(device=DEV).manual_seed(1)
    period = torch.randn(1 << 20, generator=g, device=DEV)
    fill = lambda scale: (period * scale).to(BF).repeat(-(-n // (1 << 20)))[:n].contiguous()
    p, grad = fill(0.1), fill(1e-3)
    m, v = (torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    ms, vs = torch.zeros(2, -(-n // 256), device=DEV).unbind()
    places = [(0, 1024), (2 ** 31 - 512, 2 ** 31 + 512), (2 ** 32 - 512, 2 ** 32 + 512), (2 ** 32 + 512, n)]
    old = [(p[a:b].float().cpu().numpy(), grad[a:b].float().cpu().numpy()) for a, b in places]
    args = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, grad_scale=1.0, seed=5, offset=6, step=3)
    binding.halo_adamw([p], [grad], [m], [v], m_scales=[ms], v_scales=[vs], **args)
    for (a, b), (op, og) in zip(places, old):
        k = b - a
        z = lambda: np.zeros(k, np.uint8)
        zs = lambda: np.zeros(-(-k // 256), np.float32)
        wp, wm, wv, wms, wvs = orc.adamw(op, og, z(), z(), m_scale=zs(), v_scale=zs(), bf16=True, first=a, **args)
        assert np.array_equal(p[a:b].view(torch.int16).cpu().numpy().view(np.uint16), wp), a
        for got, want in ((m, wm), (v, wv)):
            got = got[a:b].view(torch.uint8).cpu().numpy()
            assert np.array_equal(np.where(got & 127, got, 0), np.where(want & 127, want, 0)), a
        assert np.array_equal(ms[a // 256:-(-b // 256)].cpu().numpy(), wms) and np.array_equal(vs[a // 256:-(-b // 256)].cpu().numpy(), wvs)


ROWS, COLS = 66_000, 33_000            # 2^31.02 elements


def wide(seed):
    """[ROWS, COLS] of one random period of 1009 rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    period = torch.randn(1009, COLS, generator=g, device=DEV).to(BF)
    return period.repeat(-(-ROWS // 1009), 1)[:ROWS].contiguous()


def test_activation_bwd():
    e, z = wide(1), wide(2)
    ez, gb = binding.halo_activation_bwd(e, z, "silu")
    at = [0, 1, 1009, ROWS // 2, ROWS - 2, ROWS - 1]
    d = host(e[at]) * orc.slope(host(z[at]), "silu")
    within(ez[at], d, 24 * U * np.abs(host(e[at])) + HALF[BF] * np.abs(d) * (1 + 1e-5), "EZ")
    # rows repeat: every product is counted as often as its row
    times = np.bincount(np.arange(ROWS) % 1009, minlength=1009)[:, None]
    d = host(e[:1009]) * orc.slope(host(z[:1009]), "silu")
    within(gb, (times * d).sum(axis=0), (times * (24 * U * np.abs(host(e[:1009])) + column_terms(ROWS) * U * np.abs(d))).sum(axis=0), "GB")


def test_norm():
    x = wide(3)[:, :32768]                 # rows 33000 apart
    assert x.stride(0) == COLS
    y, mean, rstd = binding.halo_layer_norm_fwd(x)
    at = [0, 1009, ROWS // 2, ROWS - 1]
    want, m, r = orc.norm(host(x[at]), None, None, 1e-5, "layer")
    within(y[at], want, (HALF[BF] + 600 * U) * np.abs(want) + 600 * U, "Y")
    within(rstd[at], r, 600 * U * r, "rstd")
    ex, gw, gb = binding.halo_layer_norm_bwd(y, x, mean, rstd)
    M, R = host(mean[at]), host(rstd[at])
    want, _, _ = orc.norm_grad(host(y[at]), host(x[at]), M, R, None, None, "layer")
    # y is xh itself: what is left of it behind the norm is its rounding, a difference of numbers of the size of y
    within(ex[at], want, 2000 * U * np.abs(host(y[at])) + 2000 * U + HALF[BF] * np.abs(want), "EX")
    # the same rows, the same results
    for t in (y, ex):
        assert torch.equal(t[ROWS - 1], t[(ROWS - 1) % 1009])


def test_product():
    g = torch.Generator(device=DEV).manual_seed(4)
    A = torch.randint(-127, 128, (ROWS, 32), generator=g, device=DEV, dtype=torch.int8)
    B = torch.randint(-127, 128, (COLS, 32), generator=g, device=DEV, dtype=torch.int8)
    cs = torch.full((COLS,), 1e-5, device=DEV)
    res = wide(5)
    C, Z = binding.halo_gemm_i8_epilogue(A, B, col_scale=cs, activation="gelu", residual=res, out_dtype=BF, want_z=True)
    at = [0, 255, 256, 32768, ROWS // 2, ROWS - 2, ROWS - 1]
    y, z = orc.product(A[at].cpu().numpy(), B.cpu().numpy(), None, cs.cpu().numpy(), None, "gelu", host(res[at]))
    act = orc.act(z, "gelu")
    within(Z[at], z, 4 * U * np.abs(z) + HALF[BF] * np.abs(z) * (1 + 1e-5), "Z")
    within(C[at], y, 6 * U * np.abs(z) + act_bound(z, act, "gelu", BF) + U * np.abs(y) + HALF[BF] * np.abs(y) * (1 + 1e-5), "C")


@pytest.mark.parametrize("which", ["C", "Z", "residual", "A", "B"])
def test_product_of_far_apart_rows(which):
    """Rows 2^22 + 8 elements (codes: 2^24 + 16) apart: a tile's rows do not fit one buffer."""
    far = {"A": 2 ** 24 + 16, "B": 2 ** 24 + 16}.get(which, 2 ** 22 + 8)

    def place(t, name):
        if name != which:
            return t
        b = torch.zeros(t.shape[0], far, dtype=t.dtype, device=DEV)[:, :t.shape[1]]
        return b.copy_(t)

    g = torch.Generator(device=DEV).manual_seed(6)
    A, B = (torch.randint(-127, 128, s, generator=g, device=DEV, dtype=torch.int8) for s in ((21, 64), (40, 64)))
    res = torch.randn(21, 40, generator=g, device=DEV)
    args = dict(col_scale=torch.full((40,), 1e-4, device=DEV), activation="silu")
    empty = lambda: torch.zeros(21, 40, device=DEV)
    want = binding.halo_gemm_i8_epilogue(A, B, residual=res, out=empty(), Z=empty(), **args)
    got = binding.halo_gemm_i8_epilogue(place(A, "A"), place(B, "B"), residual=place(res, "residual"), out=place(empty(), "C"), Z=place(empty(), "Z"),
                                        **args)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
