"""Pins of oracle/around_oracle.py on the CPU: against published values, other implementations, and differences."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as orc

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def test_random_bits():
    """Known answers of Philox4x32-10 (Salmon et al., the vectors of all zeros and all ones)."""
    zero = orc.philox([[0], [0], [0], [0]], 0)
    assert [int(w[0]) for w in zero] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = orc.philox([[0xFFFFFFFF]] * 4, 2 ** 64 - 1)
    assert [int(w[0]) for w in ones] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    u = orc.random16(100_000, 3, 1, 5, 7)
    assert u.min() >= 0 and u.max() < 65536 and abs(u.mean() / 65535 - 0.5) < 5 * 0.2887 / np.sqrt(1e5)
    assert not np.array_equal(u, orc.random16(100_000, 3, 2, 5, 7)) and not np.array_equal(u, orc.random16(100_000, 2, 1, 5, 7))


def test_e4m3_table():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(orc.e4m3_decode(np.arange(256)), t, equal_nan=True)
    assert orc.E4M3[-1] == 448 and orc.E4M3[1] == 2.0 ** -9 and (np.diff(orc.E4M3) > 0).all()


@pytest.mark.parametrize("name", ACTS)
def test_activations(name):
    z = torch.linspace(-9, 9, 4001, dtype=torch.float64, requires_grad=True)
    f = {"none": lambda x: x * 1, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "gelu_tanh": lambda x: torch.nn.functional.gelu(x, approximate="tanh")}[name]
    y = f(z)
    y.sum().backward()
    np.testing.assert_allclose(orc.act(z.detach().numpy(), name), y.detach().numpy(), rtol=1e-9, atol=1e-12)
    np.testing.assert_allclose(orc.slope(z.detach().numpy(), name), z.grad.numpy(), rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm(kind):
    """Against torch's gradients, and against differences of the forward pass."""
    rng = np.random.default_rng(0)
    x, w, b, e, base = rng.normal(size=(5, 7)), rng.normal(size=7), rng.normal(size=7), rng.normal(size=(5, 7)), rng.normal(size=(5, 7))
    y, mean, rstd = orc.norm(x, w, b, 1e-3, kind)
    tx, tw, tb = (torch.tensor(v, requires_grad=True) for v in (x, w, b))
    ty = torch.nn.functional.layer_norm(tx, (7,), tw, tb, 1e-3) if kind == "layer" else torch.nn.functional.rms_norm(tx, (7,), tw, 1e-3) + tb
    np.testing.assert_allclose(y, ty.detach().numpy(), rtol=1e-10, atol=1e-12)
    ty.backward(torch.tensor(e))
    ex, gw, gb = orc.norm_grad(e, x, mean, rstd, w, base, kind)
    for got, want in ((ex - base, tx.grad), (gw, tw.grad), (gb, tb.grad)):
        np.testing.assert_allclose(got, want.numpy(), rtol=1e-9, atol=1e-12)
    h, i, j = 1e-6, 3, 4
    up, down = x.copy(), x.copy()
    up[i, j] += h
    down[i, j] -= h
    d = ((orc.norm(up, w, b, 1e-3, kind)[0] - orc.norm(down, w, b, 1e-3, kind)[0]) * e).sum() / (2 * h)
    assert abs(d - (ex - base)[i, j]) < 1e-7


def test_adamw_is_torch_s():
    """fp32 against torch.optim.AdamW in 64 bits: over a step each operation is off by 2^-24, and eight of them follow one another."""
    rng = np.random.default_rng(1)
    p0 = rng.normal(size=1000).astype(np.float32)
    t = torch.tensor(p0.astype(np.float64), requires_grad=True)
    opt = torch.optim.AdamW([t], lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    p, m, v = p0, np.zeros(1000, np.float32), np.zeros(1000, np.float32)
    for step in range(1, 6):
        g = rng.normal(size=1000).astype(np.float32)
        t.grad = torch.tensor(g.astype(np.float64) * 0.5)
        opt.step()
        p, m, v, _, _ = orc.adamw(p, g, m, v, step=step, lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1, grad_scale=0.5)
        np.testing.assert_allclose(p, t.detach().numpy(), rtol=5 * 8 * 2.0 ** -24, atol=5 * 1e-3 * 16 * 2.0 ** -24)


@pytest.mark.parametrize("square", [False, True])
def test_codes_are_right_on_average(square):
    """Of many draws the mean is the number itself, of v its square; a number that e4m3 has stays; no v but 0 becomes 0."""
    rng = np.random.default_rng(2)
    x = np.abs(rng.normal(size=256)).astype(np.float32) ** 3
    x[0], x[1], x[2] = 4.48, 0.0, 1e-6
    draws = 4000
    total = np.zeros(256)
    for k in range(draws):
        c, s = orc.codes_of(x, rng.integers(0, 65536, 256), square)
        value = orc.e4m3_decode(c).astype(np.float64) * s[0]
        total += value ** 2 if square else value
    want = x.astype(np.float64) ** (2 if square else 1)
    q = x / x.max() * 448
    gap = np.where(q < 2.0 ** -6, 2.0 ** -9, 2.0 ** (np.floor(np.log2(np.maximum(q, 2.0 ** -9))) - 3)) * x.max() / 448
    spread = gap / 2 * ((2 * x + gap) if square else 1)                 # of one draw, at most
    # a root below e4m3's first step, 2^-9 of the scale, is always kept as that step (nothing between 0 and it, and never 0): by the
    # definition its mean is that step's square, not its own, so these elements (1e-6 and a few cubes) are not in the comparison
    many = np.full(256, True) if not square else (q >= 2.0 ** -9) | (x == 0)
    assert many.sum() > 240 and (not square or not many[2])
    assert (np.abs(total / draws - want) <= 6 * spread / np.sqrt(draws) + 1e-6 * want + 2 ** -16 * spread)[many].all()
    top = x.argmax()
    c, s = orc.codes_of(x, np.full(256, 65535), square)
    assert c[top] == 126 and c[1] == 0 and (not square or c[2] == 1)
    assert s[0] == np.float32(x[top]) / np.float32(448)


def test_codes_at_the_ends():
    for square in (False, True):
        z = np.zeros(300, np.float32)
        c, s = orc.codes_of(z, np.zeros(300, np.int64), square)
        assert not c.any() and (s == np.float32(2.0 ** -110) / np.float32(448)).all()
        z[5], z[260] = np.inf, 1.0
        c, s = orc.codes_of(z, np.zeros(300, np.int64), square)
        assert (c[:256] == 127).all() and s[0] == np.inf and c[260] == 126 and (c[261:] == 0).all()
        z[5] = np.nan
        c, s = orc.codes_of(z, np.zeros(300, np.int64), square)
        assert (c[:256] == 127).all() and np.isnan(s[0]) and c[260] == 126


def test_states_in_8_bits_follow():
    """Over many steps of one gradient distribution, v in 8 bits has v's mean: to nearest it would not move from where it starts."""
    rng = np.random.default_rng(3)
    n, steps = 4096, 1200
    b2 = 0.99
    z8 = lambda: np.zeros(n, np.uint8)
    m, v, ms, vs = z8(), z8(), np.zeros(n // 256, np.float32), np.zeros(n // 256, np.float32)
    p = np.zeros(n, np.float32)
    mean8 = np.zeros(n)
    for step in range(1, steps + 1):
        g = rng.normal(size=n).astype(np.float32)
        p, m, v, ms, vs = orc.adamw(p, g, m, v, step=step, lr=0.0, betas=(0.9, b2), eps=1e-8, weight_decay=0.0, grad_scale=1.0, seed=9,
                                    m_scale=ms, v_scale=vs)
        if step > steps // 2:
            mean8 += (orc.e4m3_decode(v).astype(np.float64) * np.repeat(vs, 256)) ** 2
    # v's own mean is 1; of the time average over 600 steps with a memory of 100, over 4096 elements, the error is far below 2 %
    assert abs(mean8.mean() / (steps // 2) - 1) < 0.02
