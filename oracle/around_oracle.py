"""Plain forms of what stands around a layer's products, in 64 bits, and of the AdamW step with states in 8 bits, bit for bit in fp32.

Written from the formulas in include/halo.h; shares no code with the kernels.  Test infrastructure only.
"""
import numpy as np
from scipy.special import erfc

F = np.float32


# ---- activations and their slopes, 64 bits ----
def act(z, name):
    z = np.asarray(z, np.float64)
    if name == "none":
        return z
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "gelu":
        return z * 0.5 * erfc(-z / np.sqrt(2))
    with np.errstate(over="ignore"):
        if name == "silu":
            return z / (1 + np.exp(-z))
        return z / (1 + np.exp(-2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))


def slope(z, name):
    z = np.asarray(z, np.float64)
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if name == "gelu":
        return 0.5 * erfc(-z / np.sqrt(2)) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    k = 1.0 if name == "silu" else 2 * np.sqrt(2 / np.pi)
    u, du = (z, 1.0) if name == "silu" else (k * (z + 0.044715 * z ** 3), k * (1 + 3 * 0.044715 * z ** 2))
    with np.errstate(over="ignore"):
        p, q = 1 / (1 + np.exp(-u)), 1 / (1 + np.exp(u))
    return p + z * p * q * du


# ---- products and norms, 64 bits ----
def product(A, B, row_scale, col_scale, bias, name, residual):
    z = A.astype(np.float64) @ B.astype(np.float64).T
    z = z * (1.0 if row_scale is None else row_scale.astype(np.float64)[:, None]) * (1.0 if col_scale is None else col_scale.astype(np.float64))
    if bias is not None:
        z = z + bias.astype(np.float64)
    y = act(z, name)
    return (y if residual is None else y + residual.astype(np.float64)), z


def norm(x, w, b, eps, kind):
    x = x.astype(np.float64)
    mean = x.mean(axis=1) if kind == "layer" else np.zeros(len(x))
    d = x - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(axis=1) + eps)
    y = d * rstd[:, None] * (1.0 if w is None else w.astype(np.float64)) + (0.0 if b is None else b.astype(np.float64))
    return y, mean, rstd


def norm_grad(e, x, mean, rstd, w, base, kind):
    """mean and rstd as they were saved."""
    e, x, rstd = e.astype(np.float64), x.astype(np.float64), rstd.astype(np.float64)[:, None]
    xh = (x - (0.0 if kind == "rms" else mean.astype(np.float64)[:, None])) * rstd
    d = e * (1.0 if w is None else w.astype(np.float64))
    ex = d - xh * (d * xh).mean(axis=1, keepdims=True)
    if kind == "layer":
        ex = ex - d.mean(axis=1, keepdims=True)
    ex = ex * rstd + (0.0 if base is None else base.astype(np.float64))
    return ex, (e * xh).sum(axis=0), e.sum(axis=0)


# ---- e4m3 ----
def e4m3_values():
    """Values of the codes 0 .. 126 (1 sign, 4 exponent with bias 7, 3 mantissa bits, no infinity; 127 is NaN)."""
    v = np.empty(127)
    for c in range(127):
        e, f = c >> 3, c & 7
        v[c] = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
    return v


E4M3 = e4m3_values()


def e4m3_decode(codes):
    c = codes.astype(np.int64)
    v = np.where((c & 127) == 127, np.nan, E4M3[np.minimum(c & 127, 126)])
    return np.where(c & 128, -v, v).astype(F)


# ---- random bits ----
def philox(counter, key):
    """Philox4x32-10; counter: four arrays of 32-bit values, key: 64 bits.  Returns four arrays."""
    x = [np.asarray(c, np.uint64) for c in counter]
    low = np.uint64(0xFFFFFFFF)
    for r in range(10):
        k0, k1 = np.uint64(((key & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF), np.uint64(((key >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> np.uint64(32)) ^ x[1] ^ k0, q & low, (p >> np.uint64(32)) ^ x[3] ^ k1, p & low]
    return x


def random16(n, tensor, kind, seed, offset, first=0):
    """Of the elements from `first` on, a multiple of 8."""
    g = np.arange((n + 7) // 8, dtype=np.uint64) + np.uint64(first // 8)
    full = lambda v: np.full(g.shape, v & 0xFFFFFFFF, np.uint64)
    w = philox([g & np.uint64(0xFFFFFFFF), full(4 * tensor + kind), full(offset), full((offset >> 32) & 0xFFFFFFFF)], seed)
    halves = [(w[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for j in range(8)]
    return np.stack(halves, axis=1).reshape(-1)[:n].astype(np.int64)


# ---- AdamW ----
def to_bf16(x):
    """fp32 -> bf16 bits, to nearest, ties to even."""
    b = np.asarray(x, F).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r).astype(np.uint16)


def from_bf16(bits):
    return (bits.astype(np.uint32) << 16).view(F)


def codes_of(x, u, square):
    """x fp32 [n] (m, or the root of v) -> (codes uint8, scales fp32): q between its neighbours, in fp32 step by step."""
    n = len(x)
    blocks = -(-n // 256)
    padded = np.zeros(blocks * 256, F)
    padded[:n] = x
    with np.errstate(invalid="ignore", over="ignore"):
        most = np.abs(padded).reshape(blocks, 256).max(axis=1)          # NaN where there is one
        bad = ~np.isfinite(most)
        most = np.where(bad, most, np.maximum(most, F(2.0 ** -110))).astype(F)
        scale = (most / F(448)).astype(F)
        inverse = (F(448) / most).astype(F)
        q = np.minimum((np.abs(x) * np.repeat(inverse, 256)[:n]).astype(F), F(448))
    bad_of = np.repeat(bad, 256)[:n]
    q = np.where(bad_of, F(0), q)
    table = E4M3.astype(F)
    c = np.searchsorted(table, q, side="right") - 1                     # the code at or below q
    lo = table[c]
    hi = np.append(table, F(480))[c + 1]
    if square:
        up = (((q - lo).astype(F) * (q + lo).astype(F)).astype(F) * F(65536)) > u.astype(F) * ((hi - lo) * (hi + lo)).astype(F)
    else:
        up = (q - lo).astype(F) * F(65536) > u.astype(F) * (hi - lo).astype(F)
    c = c + up
    if square:
        c = np.where((c == 0) & (x > 0), 1, c)
    c = np.where(x < 0, c | 128, c)
    return np.where(bad_of, 127, c).astype(np.uint8), scale


def adamw(p, g, m, v, *, step, lr, betas, eps, weight_decay, grad_scale, tensor=0, seed=0, offset=0, m_scale=None, v_scale=None,
          bf16=False, first=0):
    """One tensor (flat).  p, g fp32 values; m, v fp32, or uint8 codes with their scales; bf16: p comes back as bf16 bits, rounded at
    random; first: the first element's place in the tensor.  Returns (p, m, v, m_scale, v_scale)."""
    b1, b2 = betas
    n, o = len(p), (offset + step) % 2 ** 64
    r1, r2 = F(1 - b1), F(1 - b2)
    decay, rate, root_by = F(1 - lr * weight_decay), F(lr / (1 - b1 ** step)), F(1 / np.sqrt(1 - b2 ** step))
    eight = m.dtype == np.uint8
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        if eight:
            m = e4m3_decode(m) * np.repeat(m_scale, 256)[:n]
            v = e4m3_decode(v) * np.repeat(v_scale, 256)[:n]
            v = v * v
        g = g * F(grad_scale)
        m = F(b1) * m + r1 * g
        v = F(b2) * v + r2 * (g * g)
        root = np.sqrt(v)
        p = p * decay - rate * (m / (root * root_by + F(eps)))
        assert p.dtype == F and m.dtype == F and v.dtype == F
        if bf16:
            bits = (p.view(np.uint32).astype(np.uint64) + random16(n, tensor, 0, seed, o, first).astype(np.uint64)) >> np.uint64(16)
            p = np.where(np.isnan(p), 0x7FC0, bits & np.uint64(0xFFFF)).astype(np.uint16)
        if eight:
            mc, ms = codes_of(m, random16(n, tensor, 1, seed, o, first), False)
            vc, vs = codes_of(root, random16(n, tensor, 2, seed, o, first), True)
            return p, mc, vc, ms, vs
    return p, m, v, None, None
