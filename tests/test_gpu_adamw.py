"""halo_adamw: bit for bit what the oracle's fp32 steps give, in every combination of types, and graphs that take new numbers."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as orc
from paper_2501_02625_amd import binding
from tests.gpu_util import DEV, to_dev

pytestmark = pytest.mark.gpu
HYPER = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, grad_scale=0.25)


class Model:
    """Tensors of the sizes, on the host for the oracle and on the device for the library."""

    def __init__(self, sizes, param, grad, state, seed, span=6.0):
        rng = np.random.default_rng(seed)
        self.sizes, self.param, self.grad, self.state, self.seed = sizes, param, grad, state, seed
        self.p, self.g, self.m, self.v, self.ms, self.vs = [], [], [], [], [], []
        for n in sizes:
            size = (10.0 ** (-span * rng.random(-(-n // 64)))).repeat(64)[:n]
            p, g = rng.normal(size=n).astype(np.float32), (size * rng.normal(size=n)).astype(np.float32)
            g[rng.random(n) < 0.05] = 0.0
            if param == "bf16":
                p = orc.from_bf16(orc.to_bf16(p))
            if grad == "bf16":
                g = orc.from_bf16(orc.to_bf16(g))
            self.p.append(p)
            self.g.append(g)
            if state == 8:
                b = -(-n // 256)
                self.m.append(rng.integers(0, 256, n).astype(np.uint8))
                self.m[-1][(self.m[-1] & 127) == 127] = 5
                self.v.append(rng.integers(0, 127, n).astype(np.uint8))
                self.ms.append((10.0 ** (-span * rng.random(b)) / 448).astype(np.float32))
                self.vs.append((10.0 ** (-span * rng.random(b)) / 448).astype(np.float32))
            else:
                self.m.append((size * rng.normal(size=n)).astype(np.float32))
                self.v.append((size * rng.random(n)).astype(np.float32) ** 2)
                self.ms.append(None)
                self.vs.append(None)
        bf = lambda a: to_dev(orc.to_bf16(a).view(np.int16)).view(torch.bfloat16)
        code = lambda a: to_dev(a).view(torch.float8_e4m3fn) if state == 8 else to_dev(a)
        # behind every tensor lies something that is not the call's
        guard = lambda t: torch.cat([t, torch.full((64,), 3, device=DEV).to(t.dtype)])
        self.buffers = {"p": [guard(to_dev(a) if param == "fp32" else bf(a)) for a in self.p], "m": [guard(code(a).view(torch.uint8) if state == 8 else code(a)) for a in self.m],
                        "v": [guard(code(a).view(torch.uint8) if state == 8 else code(a)) for a in self.v]}
        cut = lambda name, as8: [(b[:n].view(torch.float8_e4m3fn) if as8 and state == 8 else b[:n]) for b, n in zip(self.buffers[name], sizes)]
        self.dp, self.dm, self.dv = cut("p", False), cut("m", True), cut("v", True)
        self.dg = [bf(a) if grad == "bf16" else to_dev(a) for a in self.g]
        self.dmaster = [to_dev(a) for a in self.p] if param == "master" else None
        self.dms, self.dvs = ([to_dev(a) for a in x] if state == 8 else None for x in (self.ms, self.vs))

    def call(self, **more):
        binding.halo_adamw(self.dp, self.dg, self.dm, self.dv, masters=self.dmaster, m_scales=self.dms, v_scales=self.dvs, **more)

    def expect(self, **more):
        for t in range(len(self.sizes)):
            r = orc.adamw(self.p[t], self.g[t], self.m[t], self.v[t], tensor=t, m_scale=self.ms[t], v_scale=self.vs[t], bf16=self.param == "bf16", **more)
            p, self.m[t], self.v[t], self.ms[t], self.vs[t] = r
            self.p[t] = orc.from_bf16(p) if self.param == "bf16" else p

    def compare(self, what=""):
        same = lambda got, want: np.array_equal(got, want, equal_nan=got.dtype.kind == "f")
        for t, n in enumerate(self.sizes):
            where = "%s tensor %d of %d elements: " % (what, t, n)
            if self.param == "fp32":
                assert same(self.dp[t].cpu().numpy(), self.p[t]), where + "p"
            else:
                bits = self.dp[t].view(torch.int16).cpu().numpy().view(np.uint16)
                assert same(bits, orc.to_bf16(self.p[t])), where + "p"
            if self.dmaster:
                assert same(self.dmaster[t].cpu().numpy(), self.p[t]), where + "master"
            if self.state == 8:
                for name, d, w in (("m", self.dm, self.m), ("v", self.dv, self.v)):
                    got = d[t].view(torch.uint8).cpu().numpy()
                    got, want = (np.where(a & 127, a, 0) for a in (got, w[t]))           # -0 is 0
                    assert same(got, want), where + name + " %s" % np.argwhere(got != want)[:3].tolist()
                for name, d, w in (("m_scale", self.dms, self.ms), ("v_scale", self.dvs, self.vs)):
                    assert same(d[t].cpu().numpy(), w[t]), where + name
            else:
                assert same(self.dm[t].cpu().numpy(), self.m[t]) and same(self.dv[t].cpu().numpy(), self.v[t]), where + "states"
            for name, b in self.buffers.items():
                assert (b[t][n:].float() == 3).all(), where + "written behind " + name


RAGGED = [1, 2, 7, 8, 9, 255, 256, 257, 2047, 2048, 2049, 0, 5000, 100_003]


@pytest.mark.parametrize("state", [32, 8])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("param", ["fp32", "bf16", "master"])
def test_steps(param, grad, state):
    """Three steps in a row, each from what the one before left."""
    m = Model(RAGGED, param, grad, state, 1)
    for step in (1, 2, 3):
        more = dict(HYPER, step=step, seed=0x123456789ABCDEF0, offset=2 ** 40 + 5)
        m.call(**more)
        m.expect(**more)
        m.compare("step %d:" % step)


@pytest.mark.parametrize("state", [32, 8])
def test_many_tensors(state):
    """More tensors than one launch takes."""
    rng = np.random.default_rng(2)
    sizes = [int(n) for n in rng.integers(0, 700, 130)]
    m = Model(sizes, "bf16", "bf16", state, 3)
    more = dict(HYPER, step=10, seed=7, offset=9)
    m.call(**more)
    m.expect(**more)
    m.compare()


def test_a_large_tensor():
    m = Model([3_000_001], "bf16", "bf16", 8, 4)
    more = dict(HYPER, step=1000, seed=7, offset=9)
    m.call(**more)
    m.expect(**more)
    m.compare()


@pytest.mark.parametrize("state", [32, 8])
def test_extremes(state):
    """Gradients of 0, tiny and huge, infinite and NaN; states of 0; an eps of 0 with nothing to divide by."""
    sizes = [256] * 8
    m = Model(sizes, "fp32", "fp32", state, 5)
    for t, n in enumerate(sizes):
        if state == 8:
            for x in (m.m[t], m.v[t]):
                x[:] = 0
        else:
            m.m[t][:] = 0
            m.v[t][:] = 0
        m.g[t][:] = [0.0, 1e-30, 1e-20, 1e15, 1e25, 1.0, 1.0, 1.0][t]
    m.g[5][3], m.g[6][250], m.g[7][0] = np.inf, np.nan, -np.inf
    if state == 8:
        for t in range(8):
            m.ms[t][:] = m.vs[t][:] = 0.0
            m.dms[t].zero_()
            m.dvs[t].zero_()
            m.dm[t].view(torch.uint8).zero_()
            m.dv[t].view(torch.uint8).zero_()
    else:
        for x in m.dm + m.dv:
            x.zero_()
    for d, g in zip(m.dg, m.g):
        d.copy_(to_dev(g))
    more = dict(HYPER, eps=0.0, step=1, seed=1, offset=0)
    for step in (1, 2):
        m.call(**dict(more, step=step))
        m.expect(**dict(more, step=step))
        m.compare("step %d:" % step)


@pytest.mark.parametrize("state", [32, 8])
def test_nan_parameters_stay_nan(state):
    """bf16 parameters of their own: a NaN in the parameter, in the gradient and, with any payload, in a 32-bit state."""
    m = Model([1024], "bf16", "bf16", state, 9)
    m.dp[0][3], m.dg[0][500] = float("nan"), float("nan")
    m.dp[0][700:702].view(torch.int16).fill_(0x7FFF)
    gone = {3, 500, 700, 701}
    if state == 32:
        m.dm[0][800:801].view(torch.int32).fill_(0x7FFFFFFF)
        m.dv[0][801:802].view(torch.int32).fill_(-1)
        gone |= {800, 801}
    m.call(**dict(HYPER, step=1, seed=1, offset=0))
    assert set(torch.isnan(m.dp[0].float()).nonzero()[:, 0].tolist()) == gone


def test_no_state_of_0_is_divided_by():
    """8 bits: where v is far below its block's largest, it is kept above 0, and the update stays bounded when the gradient ends."""
    n = 1024
    g = torch.full((n,), 1e-6, device=DEV)
    g[::256] = 1e3
    p, m, v = torch.zeros(n, device=DEV), *(torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    ms, vs = torch.zeros(2, 4, device=DEV)
    args = dict(lr=1.0, betas=(0.9, 0.95), eps=0.0, weight_decay=0.0, m_scales=[ms], v_scales=[vs], seed=3)
    binding.halo_adamw([p], [g], [m], [v], step=1, **args)
    assert (v.float() > 0).all()
    before = p.clone()
    for step in range(2, 20):
        g.zero_()
        binding.halo_adamw([p], [g], [m], [v], step=step, **args)
    assert torch.isfinite(p).all() and (p - before).abs().max() < 100


def test_numbers_from_the_device_and_graphs():
    """step, lr and grad_scale in device memory: a graph replayed is the steps one after another; twice, with other work between."""
    m = Model([1000, 77, 3000], "bf16", "bf16", 8, 6)
    step = torch.zeros((), dtype=torch.int64, device=DEV)
    lr, gs = torch.zeros((), device=DEV), torch.zeros(1, device=DEV)
    first = [t.clone() for t in m.dp + m.dms + m.dvs] + [t.view(torch.uint8).clone() for t in m.dm + m.dv]

    def reset():
        for t, s in zip(m.dp + m.dms + m.dvs + [x.view(torch.uint8) for x in m.dm + m.dv], first):
            t.copy_(s)

    more = dict(betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, seed=11, offset=13)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.call(step=step, lr=lr, grad_scale=gs, **more)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step += 1
        m.call(step=step, lr=lr, grad_scale=gs, **more)
    reset()
    step.zero_()
    for k in range(1, 6):
        lr.fill_(1e-3 * k)
        gs.fill_(0.5 / k)
        graph.replay()
        torch.ones(100_000, device=DEV).sum().item()
        m.expect(step=k, lr=float(np.float32(1e-3 * k)), grad_scale=float(np.float32(0.5 / k)), **more)
        m.compare("replay %d:" % k)


def test_a_gradient_of_two_parameters():
    m = Model([700, 700], "bf16", "fp32", 8, 10)
    m.g[1] = m.g[0]
    m.dg[1] = m.dg[0]
    more = dict(HYPER, step=1, seed=1, offset=0)
    m.call(**more)
    m.expect(**more)
    m.compare()


def test_two_streams():
    """Calls on two streams, each with its own tensors, at once."""
    a, b = Model([50_000], "bf16", "fp32", 8, 7), Model([60_000], "bf16", "fp32", 8, 8)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(1, 4):
        for s, m in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                m.call(**dict(HYPER, step=k, seed=1, offset=2))
    torch.cuda.synchronize()
    for m in (a, b):
        for k in range(1, 4):
            m.expect(**dict(HYPER, step=k, seed=1, offset=2))
        m.compare()


def test_a_thousand_steps_stay_finite():
    """bf16 parameters and states in 8 bits from zeros on, gradients that shrink on the way."""
    n = 4096
    want = torch.linspace(-1, 1, n, device=DEV)
    p = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    m, v = (torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    ms, vs = torch.zeros(2, n // 256, device=DEV)
    for step in range(1, 1001):
        binding.halo_adamw([p], [(p.float() - want)], [m], [v], step=step, lr=2e-3, weight_decay=0.0, m_scales=[ms], v_scales=[vs], seed=5)
    assert all(torch.isfinite(t.float()).all() for t in (p, m, v, ms, vs))


def test_refusals():
    z = lambda n=512, d=torch.float32: torch.zeros(n, dtype=d, device=DEV)
    f8 = torch.float8_e4m3fn
    ok = lambda: [z()]
    call = lambda p, g, m, v, **k: binding.halo_adamw(p, g, m, v, **dict(dict(step=1, lr=1e-3), **k))
    x = z(1024)
    for bad in (lambda: call(ok(), [], ok(), ok()), lambda: call(ok(), [z(511)], ok(), ok()), lambda: call(ok(), ok(), [z(512, f8)], ok()),
                lambda: call(ok(), ok(), [z(512, f8)], [z(512, f8)]), lambda: call(ok(), ok(), [z(512, f8)], [z(512, f8)], m_scales=[z(2)], v_scales=[z(3)]),
                lambda: call([x[::2]], ok(), ok(), ok()), lambda: call(ok() + [z(8, torch.bfloat16)], [z(), z(8)], [z(), z(8)], [z(), z(8)]),
                lambda: call(ok(), ok(), ok(), ok(), masters=[z(512, torch.bfloat16)]), lambda: call(ok(), ok(), [z(512, torch.bfloat16)], ok()),
                lambda: call(ok(), ok(), ok(), ok(), step=torch.ones((), device=DEV)), lambda: call([None], ok(), ok(), ok())):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: call(ok(), ok(), ok(), ok(), step=0), lambda: call(ok(), ok(), ok(), ok(), betas=(1.0, 0.9)), lambda: call([x[:512], x[:512]], [z(), z()], [z(), z()], [z(), z()]),
                lambda: call([x[:512], x[256:768]], [z(), z()], [z(), z()], [z(), z()]), lambda: call(ok(), ok(), ok(), ok(), masters=ok())):
        with pytest.raises(binding.HaloError):
            bad()
    with pytest.raises(TypeError):
        call([z(512, torch.float16)], ok(), ok(), ok())
    with pytest.raises(ValueError):
        call([z().cpu()], ok(), ok(), ok())
    call([], [], [], [])
