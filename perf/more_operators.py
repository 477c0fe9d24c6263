"""The work of the operators around a linear layer, as cases that can be timed and compared.

Operators:
  norm         halo_layer_norm_fwd: Y = (X - mean) rstd w + b, mean and rstd of each row (kind "rms": mean 0, no b)
  norm_grad    halo_layer_norm_bwd: with xh = (X - mean) rstd and d = E w,  E_X = base + rstd (d - mean(d) - xh mean(d xh))  (kind
               "rms": without mean(d)),  G_W = sum over the rows of E xh,  G_B = sum over the rows of E
  product      halo_gemm_i8_epilogue: z = (A B^T row_scale) col_scale + bias on INT8 codes,  C = act(z) + residual,  Z = z
  act_grad     halo_activation_bwd: E_Z = E act'(Z), G_bias = sum over the rows of E act'(Z)
  adamw        halo_adamw: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, p = p (1 - lr wd) - lr / c1 * m / (sqrt(v / c2) + eps) with
               c = 1 - b^step, of many tensors at once

Every operation of halo_adamw is one fp32 operation, rounded once, in the order of the formulas, with (1 - b), (1 - lr wd), lr / c1 and
1 / sqrt(c2) from 64 bits: on which side of a border a number falls that is rounded to 8 or 16 bits is then the same everywhere.
8-bit states of halo_adamw: each 256 elements of a tensor share two fp32 scales; m is code * scale, v is (code * scale)^2, codes e4m3.
With A the largest |m| (the largest sqrt(v)) of the 256, at least 2^-110, the scale is A / 448 and q = |m| 448 / A (at most 448) lies
between two neighbours lo <= q < hi of e4m3's values; it becomes hi where 65536 (q - lo) > u (hi - lo) and lo otherwise, for v
where 65536 (q^2 - lo^2) > u (hi^2 - lo^2), and a v that is not 0 at least 2^-9.  A bf16 parameter without a master copy in fp32
becomes the upper 16 bits of (its fp32 bits + u).  u: 16 random bits, half j % 2 (the low one first) of word (j % 8) / 2 of
Philox4x32-10 with the counter (i / 8, 4 t + kind, o mod 2^32, o / 2^32), o = offset + step, and the key (seed mod 2^32, seed / 2^32),
for element i (j = i % 8) of tensor t; kind 0: parameter, 1: m, 2: v.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
OUTLIERS = 0.001          # share of the activation's channels that are outliers, as in the layer's configurations
BLOCK = 256               # elements of a tensor that share the scales of 8-bit states
BF16, F32, F64, FP8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn


def listed():
    return [
        # The norm in front of an attention projection while one token is decoded; statistics are not kept.
        _norm("norm", 1, 4096, "bf16", "rms", stats=False, name="norm_token_1x4096"),
        # The norm in front of a layer in the forward pass of a training step: 16 sequences of 512 tokens.
        _norm("norm", 8192, 4096, "bf16", "layer", name="norm_8192x4096"),
        # Gradients of a norm whose input also goes round the layer: the residual's gradient is added (batch 4 x 512 tokens).
        _norm("norm_grad", 2048, 4096, "bf16", "rms", base=True, name="norm_grad_2048x4096"),
        # Ragged gradients in fp32: odd numbers of tokens and channels, rows in a wider buffer.
        _norm("norm_grad", 1031, 1003, "fp32", "layer", name="norm_grad_ragged_1031x1003"),
        # Decode: the output projection of one token, added to the residual stream.
        _product(1, 4096, 4096, "none", residual=True, name="product_token_1x4096x4096"),
        # Sizes that no tile divides, fp32 out, everything at once.
        _product(777, 1003, 1008, "silu", out="fp32", residual=True, keep=True, name="product_ragged_777x1003x1008"),
        # Prompts through a down-projection, added to the residual stream (batch 4 x 512 tokens).
        _product(2048, 4096, 14336, "none", residual=True, name="product_2048x4096x14336"),
        # Training forward pass through an up-projection with its activation; Z is kept for the backward pass.
        _product(8192, 14336, 4096, "gelu", keep=True, name="product_8192x14336x4096"),
        # Gradient of a small layer's activation and bias in fp32, odd sizes.
        _act(1031, 1003, "fp32", "silu", name="act_grad_ragged_1031x1003"),
        # Gradient of the up-projection's activation and bias in the training step above.
        _act(8192, 14336, "bf16", "gelu", name="act_grad_8192x14336"),
        # Fine-tuning: the low-rank adapters of a layer's projections (4 adapters of rank 16) and some vectors, all in fp32.
        _adamw("262144*20,917504*8,4096*9,1003*3", "fp32", "fp32", "fp32", name="adamw_adapters_40"),
        # Training all weights of a layer in bf16 with states in 8 bits.
        _adamw("16777216*2,4194304*2,58720256*3,4096*2", "bf16", "bf16", "8bit", name="adamw_layer_9"),
    ]


def _norm(op, rows, cols, dtype, kind, stats=True, base=False, weight="same", name=None):
    """weight: type of w and b, that of the matrices ("same") or fp32.  kind "layer" has a bias, "rms" has none."""
    c = dict(op=op, rows=rows, cols=cols, dtype=dtype, kind=kind, weight=weight)
    c.update({"stats": stats} if op == "norm" else {"base": base})
    return _named(c, name)


def _product(m, n, k, act, out="bf16", bias=True, residual=False, keep=False, name=None):
    """m tokens, n out-features, k in-features; keep: Z is returned as well."""
    return _named(dict(op="product", m=m, n=n, k=k, act=act, out=out, bias=bias, residual=residual, keep=keep), name)


def _act(rows, cols, dtype, act, name=None):
    return _named(dict(op="act_grad", rows=rows, cols=cols, dtype=dtype, act=act), name)


def _adamw(sizes, param, grad, state, name=None):
    """sizes: "elements*tensors,..."; param: "fp32", "bf16" or "master" (bf16 with a master copy in fp32); state: "fp32" or "8bit"."""
    return _named(dict(op="adamw", sizes=sizes, param=param, grad=grad, state=state), name)


def _named(c, name):
    if name:
        c["name"] = name
    return c


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def _width(rng, step=1):
    """A layer width: half of the time one of the configurations', otherwise any."""
    return rng.choice([512, 1024, 4096, 14336]) if rng.random() < 0.5 else _log(rng, 16 * step, 14336, step)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choices(["norm", "norm_grad", "product", "act_grad", "adamw"], [2, 2, 3, 1, 2])[0]
        dtype = "bf16" if rng.random() < 0.7 else "fp32"
        if op in ("norm", "norm_grad"):
            c = _norm(op, _log(rng, 1, 16384), _width(rng), dtype, rng.choice(["layer", "rms"]), stats=rng.random() < 0.7,
                      base=rng.random() < 0.5, weight=rng.choice(["same", "fp32"]))
        elif op == "product":
            c = _product(_log(rng, 1, 8192), _width(rng), _width(rng, 16), rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                         out=dtype, bias=rng.random() < 0.7, residual=rng.random() < 0.5, keep=rng.random() < 0.4)
        elif op == "act_grad":
            c = _act(_log(rng, 1, 8192), _width(rng), dtype, rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]))
        else:
            sizes = ",".join("%d*%d" % (_log(rng, 1, 1 << 23), rng.randint(1, 12)) for _ in range(rng.randint(1, 6)))
            c = _adamw(sizes, rng.choice(["fp32", "bf16", "master"]), dtype, rng.choice(["fp32", "8bit"]))
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _sizes(case):
    return [int(n) for part in case["sizes"].split(",") for n, k in [part.split("*")] for _ in range(int(k))]


def work(case):
    op = case["op"]
    if op == "adamw":
        n, b = sum(_sizes(case)), {"fp32": 4, "bf16": 2}
        blocks = sum(-(-k // BLOCK) for k in _sizes(case))
        param = {"fp32": 8, "bf16": 4, "master": 10}[case["param"]]
        state = 16 * n if case["state"] == "fp32" else 4 * n + 16 * blocks
        return {"bytes": n * (param + b[case["grad"]]) + state, "flops": 15 * n}
    if op == "product":
        m, n, k, e = case["m"], case["n"], case["k"], 2 if case["out"] == "bf16" else 4
        matrices = 1 + case["residual"] + case["keep"]
        return {"bytes": m * k + n * k + matrices * m * n * e + 4 * m + 4 * n + 4 * n * case["bias"], "flops": 2 * m * n * k}
    size, e = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
    if op == "act_grad":
        return {"bytes": size * e * (2 if case["act"] == "none" else 3) + 4 * case["cols"], "flops": 20 * size}
    vectors = case["cols"] * (2 if case["kind"] == "layer" else 1)
    we = e if case["weight"] == "same" else 4
    if op == "norm":
        return {"bytes": 2 * size * e + vectors * we + case["stats"] * 4 * case["rows"] * (2 if case["kind"] == "layer" else 1),
                "flops": 8 * size}
    return {"bytes": size * e * (3 + case["base"]) + case["cols"] * we + vectors * 4 + 8 * case["rows"], "flops": 16 * size}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _dtype(text):
    return BF16 if text == "bf16" else F32


def _rows_of(values, dtype):
    """The matrix in a buffer whose rows begin at multiples of 16 bytes, with room behind rows of odd lengths."""
    rows, cols = values.shape
    pitch = -(-cols // 8) * 8 + (0 if cols % 8 == 0 else 8)
    m = torch.zeros(rows, pitch, dtype=dtype, device=DEVICE)[:, :cols]
    return m.copy_(values)


def _activations(g, rows, cols):
    x = _normal(g, rows, cols)
    x[:, torch.randperm(cols, generator=g, device=DEVICE)[:max(1, round(OUTLIERS * cols))]] *= 50.0
    return x


def _gradient(g, rows, cols):
    """Heavy-tailed, as the layer's output gradients are."""
    chi2 = _normal(g, rows, cols).square_() + _normal(g, rows, cols).square_() + _normal(g, rows, cols).square_()
    return _normal(g, rows, cols) / (chi2 / 3).sqrt_() * 1e-3


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    s = dict(case=case)
    if op in ("norm", "norm_grad"):
        rows, cols, dtype = case["rows"], case["cols"], _dtype(case["dtype"])
        wt = dtype if case["weight"] == "same" else F32
        s["X"] = _rows_of(_activations(g, rows, cols) + 0.1, dtype)
        s["w"] = (1.0 + 0.1 * _normal(g, cols)).to(wt)
        s["b"] = (0.1 * _normal(g, cols)).to(wt) if case["kind"] == "layer" else None
        s["eps"] = 1e-5
        if op == "norm_grad":
            s["E"] = _rows_of(_gradient(g, rows, cols), dtype)
            s["base"] = _rows_of(_gradient(g, rows, cols), dtype) if case["base"] else None
            s["mean"], s["rstd"] = _statistics(s)        # kept by the forward pass
            s["mean"] = s["mean"] if case["kind"] == "layer" else None
    elif op == "product":
        m, n, k, out = case["m"], case["n"], case["k"], _dtype(case["out"])
        codes = lambda rows: (_normal(g, rows, k) * 32.0).round_().clamp_(-127, 127).to(torch.int8)
        s["A"], s["B"] = codes(m), codes(n)
        s["row_scale"] = 0.02 * (0.5 + torch.rand(m, generator=g, device=DEVICE))
        s["col_scale"] = 0.06 / k ** 0.5 * (0.5 + torch.rand(n, generator=g, device=DEVICE))
        s["bias"] = (0.5 * _normal(g, n)).to(out) if case["bias"] else None
        s["residual"] = _rows_of(2.0 * _normal(g, m, n), out) if case["residual"] else None
    elif op == "act_grad":
        dtype = _dtype(case["dtype"])
        s["E"] = _rows_of(_gradient(g, case["rows"], case["cols"]), dtype)
        s["Z"] = _rows_of(2.0 * _normal(g, case["rows"], case["cols"]), dtype)
    else:
        _prepare_adamw(s, g, seed)
    return s


def _prepare_adamw(s, g, seed):
    """Every kind of buffer is one allocation, in which each tensor begins at a multiple of 256 elements; what lies between tensors is 0.
    Parameters and states are those after some steps."""
    case, sizes = s["case"], _sizes(s["case"])
    s.update(step=seed % 5000 + 100, lr=2e-5, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, grad_scale=0.5,
             seed=seed * 0x9E3779B97F4A7C15 % 2**64, offset=seed + 2**33)
    starts, blocks = [], 0
    for n in sizes:
        starts.append(blocks * BLOCK)
        blocks += -(-n // BLOCK)
    lengths = torch.tensor([-(-n // BLOCK) for n in sizes], device=DEVICE)
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=DEVICE), lengths)              # of every block
    first = torch.tensor(starts, device=DEVICE)[tensor]
    at = (torch.arange(blocks, device=DEVICE) * BLOCK - first)[:, None] + torch.arange(BLOCK, device=DEVICE)
    inside = at < torch.tensor(sizes, device=DEVICE)[tensor][:, None]
    # of every eight elements: which tensor, and which eight of it
    s["tensor8"] = tensor[:, None].expand(blocks, BLOCK // 8).contiguous()
    s["group8"] = (at[:, ::8] // 8).contiguous()
    flat = lambda x, dtype: torch.where(inside, x, 0.0).to(dtype).reshape(-1)
    size = 10.0 ** (torch.rand(blocks, 1, generator=g, device=DEVICE) * 2 - 4)                      # of a block's gradients
    s["flat_g"] = flat(size * _normal(g, blocks, BLOCK), _dtype(case["grad"]))
    p = 0.02 * _normal(g, blocks, BLOCK)
    s["flat_p"] = flat(p, F32 if case["param"] == "fp32" else BF16)
    s["flat_master"] = flat(p, F32) if case["param"] == "master" else None
    m = 0.3 * size * _normal(g, blocks, BLOCK)
    root = size * (0.5 + torch.rand(blocks, BLOCK, generator=g, device=DEVICE))
    if case["state"] == "fp32":
        s["flat_m"], s["flat_v"] = flat(m, F32), flat(root * root, F32)
    else:
        m, root = torch.where(inside, m, 0.0), torch.where(inside, root, 0.0)
        for name, x in (("m", m), ("v", root)):
            scale = x.abs().amax(dim=1, keepdim=True) / 448
            s["flat_%s" % name] = (x / scale).clamp(-448, 448).to(FP8).reshape(-1)
            s["flat_%s_scale" % name] = scale.reshape(-1)
    views = lambda x, per=1: None if x is None else [x[a // per:a // per + -(-n // per)] for a, n in zip(starts, sizes)]
    for name in ("p", "g", "m", "v", "master"):
        s[name] = views(s["flat_" + name])
    eight = case["state"] == "8bit"
    s["m_scale"], s["v_scale"] = (views(s["flat_%s_scale" % name], BLOCK) if eight else None for name in ("m", "v"))


# ------------------------------------------------------------------------------------------------ plain forms, 32 bits
def _statistics(s):
    x = s["X"].float()
    mean = x.mean(dim=1) if s["case"]["kind"] == "layer" else torch.zeros(x.shape[0], device=DEVICE)
    d = x - mean[:, None]
    return mean, torch.rsqrt((d * d).mean(dim=1) + s["eps"])


def _plain_norm(s):
    mean, rstd = _statistics(s)
    y = (s["X"].float() - mean[:, None]) * rstd[:, None] * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    out = {"Y": y.to(s["X"].dtype)}
    if s["case"]["stats"]:
        out["rstd"] = rstd
        if s["case"]["kind"] == "layer":
            out["mean"] = mean
    return out


def _plain_norm_grad(s):
    e, layer = s["E"].float(), s["case"]["kind"] == "layer"
    xh = s["X"].float()
    if layer:
        xh = xh - s["mean"][:, None]
    xh = xh * s["rstd"][:, None]
    d = e * s["w"].float()
    ex = d - xh * (d * xh).mean(dim=1, keepdim=True)
    if layer:
        ex = ex - d.mean(dim=1, keepdim=True)
    ex = ex * s["rstd"][:, None]
    if s["base"] is not None:
        ex = ex + s["base"].float()
    out = {"EX": ex.to(s["X"].dtype), "GW": (e * xh).sum(dim=0)}
    if layer:
        out["GB"] = e.sum(dim=0)
    return out


def _act_of(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z / (1 + torch.exp(-2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))


def _slope_of(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p + z * p * (1 - p)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5
    a = 2 * (2 / math.pi) ** 0.5
    p = 1 / (1 + torch.exp(-a * (z + 0.044715 * z * z * z)))
    return p + z * p * (1 - p) * a * (1 + 3 * 0.044715 * z * z)


def _plain_product(s):
    c = s["case"]
    z = (s["A"].float() @ s["B"].float().t()) * s["row_scale"][:, None] * s["col_scale"]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act_of(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"C": y.to(_dtype(c["out"]))}
    if c["keep"]:
        out["Z"] = z.to(_dtype(c["out"]))
    return out


def _plain_act_grad(s):
    d = s["E"].float() * _slope_of(s["Z"].float(), s["case"]["act"])
    return {"EZ": d.to(s["E"].dtype), "GB": d.sum(dim=0)}


def _random16(s, kind, ints=torch.int64):
    """16 random bits for every element of the flat buffers, [blocks, 256]."""
    low = 0xFFFFFFFF
    o = s["offset"] + s["step"]
    c0, c1 = s["group8"], s["tensor8"] * 4 + kind
    c2, c3 = torch.full_like(c0, o & low), torch.full_like(c0, o >> 32)
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    halves = [h.to(ints) for c in (c0, c1, c2, c3) for h in (c & 0xFFFF, c >> 16)]
    return torch.stack(halves, dim=-1).reshape(-1, BLOCK)


def _to_8bit(s, x, kind):
    """Codes (as their values) and scales of x [blocks, 256]: m itself (kind 1) or the root of v (kind 2)."""
    most = x.abs().amax(dim=1, keepdim=True).clamp_min(2.0 ** -110)
    q = (x.abs() * (torch.full_like(most, 448.0) / most)).clamp_max(448)
    step = torch.ldexp(torch.ones_like(q), torch.frexp(q)[1].clamp_min(-5) - 4)      # between neighbours; from 2^-6 down 2^-9
    lo = torch.floor(q / step) * step
    hi = lo + step
    u = _random16(s, kind).float()
    if kind == 1:
        up = (q - lo) * 65536 > u * step
    else:
        up = (q - lo) * (q + lo) * 65536 > u * (step * (hi + lo))
    code = torch.where(up, hi, lo)
    if kind == 2:
        code = torch.where(x > 0, code.clamp_min(2.0 ** -9), code)
    return torch.where(x < 0, -code, code), most / torch.full_like(most, 448.0)


def _plain_adamw(s):
    case, (b1, b2), lr = s["case"], s["betas"], s["lr"]
    eight, shape = case["state"] == "8bit", (-1, BLOCK)
    g = s["flat_g"].float().reshape(shape) * s["grad_scale"]
    m, v = s["flat_m"].float().reshape(shape), s["flat_v"].float().reshape(shape)
    if eight:
        m, v = m * s["flat_m_scale"][:, None], (v * s["flat_v_scale"][:, None]).square()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    c1, c2 = 1 - b1 ** s["step"], 1 - b2 ** s["step"]
    root = torch.sqrt(v.double()).float()                # the nearest of 32 bits
    old = s["flat_p"] if s["flat_master"] is None else s["flat_master"]
    p = old.float().reshape(shape) * (1 - lr * s["weight_decay"]) - (lr / c1) * (m / (root * (1 / c2 ** 0.5) + s["eps"]))
    if case["param"] == "bf16":
        bits = (p.view(torch.int32) + _random16(s, 0, torch.int32)) & -65536
        p = bits.view(F32)
    s["flat_p"].copy_(p.reshape(-1))
    if s["flat_master"] is not None:
        s["flat_master"].copy_(p.reshape(-1))
    if eight:
        for name, x, kind in (("m", m, 1), ("v", root, 2)):
            code, scale = _to_8bit(s, x, kind)
            s["flat_" + name].copy_(code.reshape(-1))
            s["flat_%s_scale" % name].copy_(scale.reshape(-1))
    else:
        s["flat_m"].copy_(m.reshape(-1))
        s["flat_v"].copy_(v.reshape(-1))
    return _buffers(s)


def _buffers(s):
    """The updated parameters and states; codes of 8 bits are numbers of their own type, next to their scales."""
    names = ("flat_p", "flat_master", "flat_m", "flat_v", "flat_m_scale", "flat_v_scale")
    return {name: s[name] for name in names if s.get(name) is not None}


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "product": _plain_product, "act_grad": _plain_act_grad,
                "adamw": _plain_adamw}[op](s)
    from paper_2501_02625_amd import binding
    if op == "norm":
        y, mean, rstd = binding.halo_layer_norm_fwd(s["X"], s["w"], s["b"], eps=s["eps"], kind=c["kind"], want_stats=c["stats"])
        out = {"Y": y, "mean": mean, "rstd": rstd}
        return {name: x for name, x in out.items() if x is not None}
    if op == "norm_grad":
        ex, gw, gb = binding.halo_layer_norm_bwd(s["E"], s["X"], s["mean"], s["rstd"], s["w"], kind=c["kind"], base=s["base"],
                                                 want_gb=c["kind"] == "layer")
        return {"EX": ex, "GW": gw} if gb is None else {"EX": ex, "GW": gw, "GB": gb}
    if op == "product":
        y, z = binding.halo_gemm_i8_epilogue(s["A"], s["B"], row_scale=s["row_scale"], col_scale=s["col_scale"], bias=s["bias"],
                                             activation=c["act"], residual=s["residual"], out_dtype=_dtype(c["out"]),
                                             want_z=c["keep"])
        return {"C": y} if z is None else {"C": y, "Z": z}
    if op == "act_grad":
        ez, gb = binding.halo_activation_bwd(s["E"], s["Z"], c["act"])
        return {"EZ": ez, "GB": gb}
    binding.halo_adamw(s["p"], s["g"], s["m"], s["v"], step=s["step"], lr=s["lr"], betas=s["betas"], eps=s["eps"],
                       weight_decay=s["weight_decay"], grad_scale=s["grad_scale"], masters=s["master"], m_scales=s["m_scale"],
                       v_scales=s["v_scale"], seed=s["seed"], offset=s["offset"])
    return _buffers(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def _normal_density(z):
    return torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def _exact_act(z, act):
    """act(z) and its slope."""
    one = torch.ones_like(z)
    if act == "none":
        return z, one
    if act == "relu":
        return z.clamp_min(0), (z > 0).double()
    if act == "gelu":
        below = torch.special.erfc(-z / math.sqrt(2)) / 2
        return z * below, below + z * _normal_density(z)
    inner, slope = (z, one) if act == "silu" else (math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3),
                                                   math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2))
    p = torch.sigmoid(inner)
    return z * p, p + z * p * torch.sigmoid(-inner) * slope


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "product": _exact_product, "act_grad": _exact_act_grad,
            "adamw": _exact_adamw}[case["op"]](s)


def _exact_norm(s):
    x, layer = s["X"].double(), s["case"]["kind"] == "layer"
    mean = x.sum(dim=1, keepdim=True) / x.shape[1] if layer else torch.zeros(x.shape[0], 1, dtype=F64, device=DEVICE)
    x = x - mean
    rstd = (x.square().sum(dim=1, keepdim=True) / x.shape[1] + s["eps"]) ** -0.5
    out = {"Y": x * rstd * s["w"].double() + (s["b"].double() if layer else 0)}
    if s["case"]["stats"]:
        out.update({"mean": mean[:, 0], "rstd": rstd[:, 0]} if layer else {"rstd": rstd[:, 0]})
    return out


def _exact_norm_grad(s):
    e, x, layer = s["E"].double(), s["X"].double(), s["case"]["kind"] == "layer"
    rstd, n = s["rstd"].double()[:, None], s["X"].shape[1]
    xh = (x - s["mean"].double()[:, None] if layer else x) * rstd
    d = e * s["w"].double()
    out = {"EX": rstd * (d - xh * (d * xh).sum(dim=1, keepdim=True) / n - (d.sum(dim=1, keepdim=True) / n if layer else 0))}
    if s["base"] is not None:
        out["EX"] += s["base"].double()
    out["GW"] = (e * xh).sum(dim=0)
    if layer:
        out["GB"] = e.sum(dim=0)
    return out


def _exact_product(s):
    z = torch.mm(s["A"].double(), s["B"].double().t())           # whole numbers below 2^53
    z *= s["row_scale"].double()[:, None]
    z *= s["col_scale"].double()
    if s["bias"] is not None:
        z += s["bias"].double()
    y = _exact_act(z, s["case"]["act"])[0]
    out = {"C": y if s["residual"] is None else y + s["residual"].double()}
    if s["case"]["keep"]:
        out["Z"] = z
    return out


def _exact_act_grad(s):
    d = s["E"].double() * _exact_act(s["Z"].double(), s["case"]["act"])[1]
    return {"EZ": d, "GB": d.sum(dim=0)}


def _words(counter, key):
    """Philox4x32-10 on lists of four counters (int64 tensors of 32-bit values) and a 64-bit key."""
    x, low = list(counter), (1 << 32) - 1
    for r in range(10):
        ka, kb = ((key & low) + r * 0x9E3779B9) & low, ((key >> 32) + r * 0xBB67AE85) & low
        # 32 x 32 -> 64 bits in halves of the factor, so that nothing wraps
        def product(a, f):
            lo, hi = a * (f & 0xFFFF), a * (f >> 16)
            mid = hi + (lo >> 16)
            return mid >> 16, ((mid & 0xFFFF) << 16) | (lo & 0xFFFF)
        (h0, l0), (h1, l1) = product(x[0], 0xD2511F53), product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ ka, l1, h0 ^ x[3] ^ kb, l0]
    return x


def _exact_code(v, most, u, root):
    """The e4m3 value that stands for v / (most / 448); u: random numbers in [0, 65536).  root: v's square is what is kept in the mean."""
    q = (v.abs() * 448 / most).clamp_max(448.0)
    e = torch.floor(torch.log2(q.clamp_min(2.0 ** -9)))
    e = e + (torch.exp2(e + 1) <= q).double() - (torch.exp2(e) > q).double()          # log2 next to a power of two
    gap = torch.exp2(e.clamp_min(-6.0) - 3)
    lo = (q / gap).floor() * gap
    share = (q * q - lo * lo) / ((lo + gap).square() - lo * lo) if root else (q - lo) / gap
    code = lo + gap * (65536 * share > u)
    if root:
        code = torch.where(v > 0, code.clamp_min(2.0 ** -9), code)
    return code * torch.sign(v)


def _exact_adamw(s):
    """Tensor by tensor."""
    case, (b1, b2), t, lr, low = s["case"], s["betas"], s["step"], s["lr"], (1 << 32) - 1
    eight, o = case["state"] == "8bit", s["offset"] + s["step"]
    new = {name: x.double() for name, x in _buffers(s).items()}
    start = 0
    for k, n in enumerate(_sizes(case)):
        blocks = -(-n // BLOCK)
        part = slice(start, start + n)
        scales = slice(start // BLOCK, start // BLOCK + blocks)
        start += blocks * BLOCK
        groups = torch.arange(-(-n // 8), device=DEVICE)

        def u(kind):
            w = _words([groups, torch.full_like(groups, 4 * k + kind), torch.full_like(groups, o & low), torch.full_like(groups, o >> 32)],
                       s["seed"])
            return torch.stack([(w[j // 2] >> (16 * (j % 2))) & 0xFFFF for j in range(8)], dim=1).reshape(-1)[:n]

        spread = lambda x: x[scales].repeat_interleave(BLOCK)[:n]
        m, v, g = new["flat_m"][part], new["flat_v"][part], s["flat_g"][part].double() * s["grad_scale"]
        if eight:
            m, v = m * spread(new["flat_m_scale"]), (v * spread(new["flat_v_scale"])) ** 2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
        p = new["flat_p" if s["flat_master"] is None else "flat_master"][part]
        p = p - lr * s["weight_decay"] * p - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + s["eps"])
        if s["flat_master"] is not None:
            new["flat_master"][part] = p
        if case["param"] == "bf16":                      # towards 0 or away from it, to 8 bits of significand
            gap = torch.exp2(torch.floor(torch.log2(p.abs().clamp_min(2.0 ** -126))) - 7)
            lo = (p.abs() / gap).floor() * gap
            p = torch.sign(p) * (lo + gap * ((p.abs() - lo) / gap * 65536 + u(0) >= 65536))
        new["flat_p"][part] = p
        if not eight:
            new["flat_m"][part], new["flat_v"][part] = m, v
            continue
        for name, x, kind in (("flat_m", m, 1), ("flat_v", v.sqrt(), 2)):
            padded = torch.nn.functional.pad(x.abs(), (0, blocks * BLOCK - n)).reshape(blocks, BLOCK)
            most = padded.amax(dim=1).clamp_min(2.0 ** -110)
            new[name + "_scale"][scales] = most / 448
            new[name][part] = _exact_code(x, most.repeat_interleave(BLOCK)[:n], u(kind).double(), kind == 2)
    return new
