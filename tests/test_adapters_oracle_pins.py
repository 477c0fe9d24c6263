"""CPU pins of the oracle of dropout and of the low-rank adapters: published answers of the generator, the mask's definition element by
element, the merged-weight identity that defines an adapter, and the gradients against differences."""
import numpy as np
import pytest

from oracle import adapters_oracle as orc


@pytest.mark.parametrize("counter,key,want", [
    # known answers that the generator's authors published with it
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, want):
    assert tuple(int(w) for w in orc.philox4x32_10(counter, key)) == want


def _words(counter, key):
    """The generator in Python's integers, one counter at a time."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) % 2**32, (k[1] + 0xBB67AE85) % 2**32]
    return c


def test_mask_is_what_the_definition_says():
    rows, cols, p, seed, offset = 5, 21, 0.3, 0x123456789ABCDEF0, 2**40 + 3
    mask = orc.keep_mask(rows, cols, p, seed, offset)
    for i in range(rows):
        for j in range(cols):
            w = _words([j // 8, i, offset % 2**32, offset >> 32], [seed % 2**32, seed >> 32])[(j % 8) // 2]
            bits = w & 0xFFFF if j % 2 == 0 else w >> 16
            assert mask[i, j] == (bits >= round(0.3 * 65536))


@pytest.mark.parametrize("p", [0.05, 0.5, 0.9])
def test_mask_frequency_mean_and_independence(p):
    rows, cols = 256, 1024
    n = rows * cols
    a = orc.keep_mask(rows, cols, p, 7, 1)
    q = orc.threshold(p) / 65536
    sigma = np.sqrt(q * (1 - q) / n)
    assert abs(a.mean() - (1 - q)) < 5 * sigma
    assert np.allclose(orc.drop(np.ones((rows, cols)), p, 7, 1).mean(), 1.0, atol=5 * sigma / (1 - q))
    for other in (orc.keep_mask(rows, cols, p, 7, 2), orc.keep_mask(rows, cols, p, 8, 1), np.roll(a, 1, axis=1), np.roll(a, 1, axis=0)):
        corr = np.mean((a - (1 - q)) * (other - (1 - q))) / (q * (1 - q))
        assert abs(corr) < 5 / np.sqrt(n)


def test_probabilities_zero_and_one():
    x = np.array([[1.0, np.inf, np.nan, -2.0]])
    assert np.array_equal(orc.drop(x, 0.0, 1, 2), x, equal_nan=True)
    assert np.array_equal(orc.drop(x, 1.0, 1, 2), np.zeros_like(x))


def _case(seed, p):
    g = np.random.default_rng(seed)
    b, m, n, slots, rank = 11, 10, 9, 3, 4
    X, E, U, V = g.standard_normal((b, m)), g.standard_normal((b, n)), g.standard_normal((slots, rank, m)), g.standard_normal((slots, n, rank))
    of = np.array([0, 0, 2, 1, -1, 2, 2, 3, 0, 1, 2], dtype=np.int32)
    kw = dict(ranks=np.array([4, 1, 3]), scale=np.array([0.5, -2.0, 1.25]), p=p, seed=5, offset=6)
    return X, E, U, V, of, kw


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_merged_weight_identity(p):
    """Token by token, Y = base + drop(x) (s V U)^T and E_X = base + drop'(e (s V U))."""
    X, E, U, V, of, kw = _case(1, p)
    base_y, base_x = np.random.default_rng(3).standard_normal((11, 9)), np.random.default_rng(4).standard_normal((11, 10))
    Y, T = orc.forward(X, U, V, of, base=base_y, **kw)
    EX, GU, GV, S = orc.backward(E, X, T, U, V, of, base=base_x, **kw)
    x, f = orc.drop(X, p, 5, 6), orc.drop(np.ones_like(X), p, 5, 6)
    for t, a in enumerate(of):
        if not 0 <= a < 3:
            assert np.array_equal(Y[t], base_y[t]) and np.array_equal(EX[t], base_x[t]) and not T[t].any() and not S[t].any()
            continue
        r = kw["ranks"][a]
        W = kw["scale"][a] * V[a, :, :r] @ U[a, :r]
        assert np.allclose(Y[t], base_y[t] + W @ x[t], atol=1e-12)
        assert np.allclose(EX[t], base_x[t] + f[t] * (E[t] @ W), atol=1e-12)
    assert not GU[1, 1:].any() and not GV[1, :, 1:].any()          # beyond the rank


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_gradients_against_differences(p):
    """L = <E, Y> is linear in each of U, V and X: a central difference is exact up to rounding."""
    X, E, U, V, of, kw = _case(2, p)
    loss = lambda X, U, V: float((E * orc.forward(X, U, V, of, **kw)[0]).sum())
    _, T = orc.forward(X, U, V, of, **kw)
    EX, GU, GV, _ = orc.backward(E, X, T, U, V, of, **kw)
    for k, (array, grad) in enumerate(((X, EX), (U, GU), (V, GV))):
        for i in np.ndindex(array.shape):
            args = [X, U, V]
            value = []
            for step in (1e-3, -1e-3):
                moved = array.copy()
                moved[i] += step
                args[k] = moved
                value.append(loss(*args))
            assert abs((value[0] - value[1]) / 2e-3 - grad[i]) < 1e-9
