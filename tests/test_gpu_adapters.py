"""GPU: low-rank adapters of many requests (halo_adapters_fwd / halo_adapters_bwd) against the 64-bit oracle, through the C ABI.

Bounds, from the arithmetic, u = 2^-24, |.| element by element, K the reduction length:
  T, S        (40 + K/8) u |x| |U|^T         fp32 sums of exact products, at most one rounding per 8 of them, a few more where partial
                                             sums meet and for the factors 1/(1-p) and scale
  Y, E_X      the error of T (S) carried through |V| (|U|), plus (40 + rank) u |T| |V|^T, plus 4 u |result|; the values that the
              kernels take from fp32 into matrix instructions are split exactly
  G_U, G_V    the error of S carried through |X|, plus (40 + b/8) u |S|^T |X|   (T is an input)
bf16 outputs: one rounding to 8 significant bits (2^-8 |y|) on top."""
import numpy as np
import pytest
import torch

from oracle import adapters_oracle as orc
from paper_2501_02625_amd import binding, inputs
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def real(bits):
    return inputs.bf16_bits_to_f32(bits).astype(np.float64)


class Case:
    """Inputs on both sides.  of: adapter of every token; ranks None or a list."""

    def __init__(self, b, m, n, slots, rank, of, ranks=None, scale=True, p=0.0, base=True, odt=torch.float32, seed=1):
        g = np.random.default_rng(seed)
        self.b, self.m, self.n, self.slots, self.rank, self.p, self.odt = b, m, n, slots, rank, p, odt
        bits = lambda *shape, std=1.0: inputs.f32_to_bf16_bits((g.standard_normal(shape) * std).astype(np.float32))
        self.X, self.E = bits(b, m), bits(b, n, std=0.5)
        self.U, self.V = bits(slots, rank, m, std=m ** -0.5), bits(slots, n, rank, std=0.3)
        self.of = np.asarray(of, dtype=np.int32)
        self.ranks = None if ranks is None else np.asarray(ranks, dtype=np.int32)
        self.scale = (g.standard_normal(slots) + 1.5).astype(np.float32) if scale else None
        self.seed, self.offset = int(g.integers(2**63)), int(g.integers(2**62))
        def make_base(cols):
            x = g.standard_normal((b, cols)).astype(np.float32)
            return real(inputs.f32_to_bf16_bits(x)).astype(np.float32) if odt == torch.bfloat16 else x
        self.base_y, self.base_x = (make_base(n), make_base(m)) if base else (None, None)

    def kw(self):
        """Arguments of the binding."""
        dev = lambda a: None if a is None else gu.to_dev(a)
        return dict(ranks=dev(self.ranks), scale=dev(self.scale), dropout_p=self.p, seed=self.seed, offset=self.offset, out_dtype=self.odt)

    def oracle_kw(self):
        return dict(ranks=self.ranks, scale=self.scale, p=self.p, seed=self.seed, offset=self.offset)

    def dev_base(self, a):
        return None if a is None else gu.to_dev(a).to(self.odt)

    def run(self):
        X, E, U, V = (gu.bits_to_dev(a) for a in (self.X, self.E, self.U, self.V))
        of = gu.to_dev(self.of)
        Y, T = binding.halo_adapters_fwd(X, U, V, of, base=self.dev_base(self.base_y), **self.kw())
        EX, GU, GV = binding.halo_adapters_bwd(E, X, T, U, V, of, base=self.dev_base(self.base_x), **self.kw())
        torch.cuda.synchronize()
        return Y, T, EX, GU, GV

    def check(self, Y, T, EX, GU, GV):
        X, E, U, V = (real(a) for a in (self.X, self.E, self.U, self.V))
        kw = self.oracle_kw()
        y, t = orc.forward(X, U, V, self.of, base=self.base_y, **kw)
        Td = T.cpu().numpy().astype(np.float64)
        ex, gu_, gv, s = orc.backward(E, X, Td, U, V, self.of, base=self.base_x, **kw)
        # the same sums of absolute values
        aX, aE, aU, aV = (np.abs(a) for a in (X, E, U, V))
        akw = dict(kw, scale=None if self.scale is None else np.abs(self.scale))
        ay, at = orc.forward(aX, aU, aV, self.of, **akw)
        aex, agu, agv, as_ = orc.backward(aE, aX, np.abs(Td), aU, aV, self.of, **akw)
        et, es = (40 + self.m / 8) * U32 * at, (40 + self.n / 8) * U32 * as_
        within(T, t, et, "T")
        # errors of T and S carried on: linear in T (S), and |T| <= at
        within(Y, y, ((40 + self.m / 8) + (40 + self.rank)) * U32 * ay + self.out_bound(y), "Y")
        within(EX, ex, ((40 + self.n / 8) + (40 + self.rank)) * U32 * aex + self.out_bound(ex), "EX")
        within(GU, gu_, ((40 + self.n / 8) + (40 + self.b / 8)) * U32 * agu, "GU")
        within(GV, gv, (40 + self.b / 8) * U32 * agv, "GV")

    def out_bound(self, y):
        return (4 * U32 + (2.0 ** -8 if self.odt == torch.bfloat16 else 0.0)) * np.abs(y)


def within(got, want, bound, what):
    g = got.float().cpu().numpy().astype(np.float64)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bad = ~(np.abs(g - want) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d outside the bound; first at %s: got %r want %r bound %r"
                             % (what, int(bad.sum()), want.size, i, g[i], want[i], bound[i]))


def runs(b, slots, length):
    """Tokens in runs of `length` with the adapters in turn; the last of every four runs has none."""
    a = [(i // length) % (slots + 1) for i in range(b)]
    return [-1 if x == slots else x for x in a]


def scattered(b, slots, seed=3):
    return np.random.default_rng(seed).integers(-1, slots, b)


@pytest.mark.parametrize("b,m,n,slots,rank", [
    (1, 8, 8, 1, 8), (1, 4096, 1024, 8, 16), (2, 520, 264, 2, 24), (15, 64, 136, 3, 16), (16, 1000, 1016, 1, 64), (17, 72, 40, 5, 128),
    (31, 256, 2056, 2, 32), (33, 2048, 64, 40, 8), (64, 512, 512, 64, 16), (65, 24, 1336, 4, 40), (130, 1032, 520, 3, 64),
    (257, 128, 392, 7, 112), (600, 520, 1000, 2, 48), (1025, 264, 256, 9, 72),
])
@pytest.mark.parametrize("odt,p", [(torch.float32, 0.0), (torch.bfloat16, 0.1)])
def test_sizes_and_orders(b, m, n, slots, rank, odt, p):
    for of in (runs(b, slots, max(1, b // 3)), scattered(b, slots)):
        c = Case(b, m, n, slots, rank, of, p=p, odt=odt, seed=b + m)
        c.check(*c.run())


@pytest.mark.parametrize("b,m,n,slots,rank,length", [
    (1024, 72, 4104, 3, 8, 100), (1100, 136, 1000, 70, 24, 1), (1500, 520, 520, 9, 56, 37), (2100, 264, 2056, 4, 104, 700),
    (3000, 2056, 72, 1, 16, 3000), (4100, 640, 136, 2, 40, 1300), (2048, 512, 8, 12, 128, 5),
])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_many_tokens(b, m, n, slots, rank, length, p):
    """Tiles with one adapter, at requests' borders and with more adapters than workgroups that share them; adapters with several segments,
    whole ones and the last, which is shorter; reductions that end inside a step."""
    c = Case(b, m, n, slots, rank, runs(b, slots, length), ranks=[rank - (5 * s) % rank for s in range(slots)], p=p, seed=b + n)
    c.check(*c.run())


@pytest.mark.parametrize("ranks", [[1, 16, 7, 0, 9], [16, 16, 16, 16, 16], [0, 0, 0, 0, 0], [3, -4, 15, 99, 8]])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_ranks_of_their_own(ranks, p):
    c = Case(97, 200, 344, 5, 16, scattered(97, 5), ranks=ranks, p=p)
    out = c.run()
    c.check(*out)
    clamped = np.clip(ranks, 0, 16)
    for a in range(5):
        assert not out[3][a, clamped[a]:].any() and not out[4][a, :, clamped[a]:].any()


@pytest.mark.parametrize("rank", [64, 128, 104])
def test_large_ranks_of_their_own(rank):
    ranks = [rank, 1, rank - 1, 33, 17, 64]
    c = Case(210, 328, 152, 6, rank, scattered(210, 6), ranks=ranks, p=0.2)
    c.check(*c.run())


@pytest.mark.parametrize("of", [[-1] * 40, [7] * 40, [2] * 40, [-2**31, 2**31 - 1, 3, 0] * 10])
def test_tokens_without_an_adapter(of):
    c = Case(40, 96, 200, 3, 16, of, odt=torch.bfloat16)
    out = c.run()
    c.check(*out)
    none = [i for i, a in enumerate(of) if not 0 <= a < 3]
    assert torch.equal(out[0][none], c.dev_base(c.base_y)[none]) and torch.equal(out[2][none], c.dev_base(c.base_x)[none])
    for a in range(3):
        if a not in of:
            assert not out[3][a].any() and not out[4][a].any()


@pytest.mark.parametrize("scale", [True, False])
@pytest.mark.parametrize("base", [True, False])
@pytest.mark.parametrize("odt", [torch.float32, torch.bfloat16])
def test_without_scale_or_base(scale, base, odt):
    c = Case(50, 136, 72, 4, 8, scattered(50, 4), scale=scale, base=base, odt=odt, p=0.5)
    c.check(*c.run())


@pytest.mark.parametrize("b,rank", [(9, 16), (200, 64)])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_what_is_not_used_may_hold_anything(b, rank, p):
    """NaN and infinities beyond the ranks, in pool places without tokens, in the rows of tokens without an adapter and in dropped
    elements reach nothing."""
    c = Case(b, 264, 336, 4, rank, [[0, 1, -1, 1, 3][i % 5] for i in range(b)], ranks=[rank - 3, 5, rank, rank], p=p, base=True)
    bad = np.array([0x7FC0, 0x7F80, 0xFF80, 0xFFC1], dtype=np.uint16)
    fill = lambda shape: bad[np.random.default_rng(0).integers(0, 4, shape)]
    clean = {k: getattr(c, k).copy() for k in ("X", "E", "U", "V")}
    for a, r in enumerate(c.ranks):
        c.U[a, r:], c.V[a, :, r:] = fill(c.U[a, r:].shape), fill(c.V[a, :, r:].shape)
    c.U[2], c.V[2] = fill(c.U[2].shape), fill(c.V[2].shape)
    none = np.flatnonzero(c.of < 0)
    c.X[none], c.E[none] = fill((len(none), c.m)), fill((len(none), c.n))
    if p:
        dropped = ~orc.keep_mask(b, c.m, p, c.seed, c.offset)
        c.X[dropped] = fill(int(dropped.sum()))
    out = c.run()
    for k, v in clean.items():
        setattr(c, k, v)
    c.check(*out)


def test_infinities_and_nan_stay_in_their_token_and_column():
    c = Case(48, 128, 160, 2, 16, [0] * 20 + [1] * 28, odt=torch.float32)
    clean = c.run()
    c.X[5, 17], c.E[30, 9] = 0x7F80, 0x7FC0
    Y, T, EX, GU, GV = c.run()
    keep = [i for i in range(48) if i != 5]
    assert torch.equal(Y[keep], clean[0][keep]) and not torch.isfinite(T[5]).any()
    keep = [i for i in range(48) if i != 30]
    assert torch.equal(EX[keep], clean[2][keep]) and torch.isnan(EX[30]).all()
    assert torch.equal(GU[0][:, :17], clean[3][0][:, :17]) and torch.equal(GU[0][:, 18:], clean[3][0][:, 18:])
    assert not torch.isfinite(GU[0][:, 17]).any() and torch.isnan(GU[1]).all()
    assert torch.isnan(GV[1][9]).all() and torch.equal(GV[1][:9], clean[4][1][:9]) and torch.equal(GV[1][10:], clean[4][1][10:])


@pytest.mark.parametrize("odt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b", [3, 77])
def test_strides_and_guards(b, odt):
    """Every matrix a column range of a wider one: nothing beside it is read into a result or written."""
    c = Case(b, 120, 88, 3, 24, scattered(b, 3), p=0.25, odt=odt)
    want = c.run()
    pads = dict(X=(c.X, 16, 136 + 24), E=(c.E, 8, 88 + 40))
    wide = {}
    for k, (bits, lo, cols) in pads.items():
        buf = torch.full((b, cols), float("nan"), dtype=torch.bfloat16, device=gu.DEV)
        buf[:, lo:lo + bits.shape[1]] = gu.bits_to_dev(bits)
        wide[k] = buf[:, lo:lo + bits.shape[1]]
    def room(cols, fill=float("nan")):
        buf = torch.full((b + 2, cols + 32), fill, dtype=odt, device=gu.DEV)
        return buf, buf[1:b + 1, 16:16 + cols]
    by, base_y = room(c.n); base_y.copy_(c.dev_base(c.base_y))
    bx, base_x = room(c.m); base_x.copy_(c.dev_base(c.base_x))
    oy, Y = room(c.n, 7.0); ox, EX = room(c.m, 7.0)
    U, V, of = gu.bits_to_dev(c.U), gu.bits_to_dev(c.V), gu.to_dev(c.of)
    _, T = binding.halo_adapters_fwd(wide["X"], U, V, of, base=base_y, Y=Y, **c.kw())
    _, GU, GV = binding.halo_adapters_bwd(wide["E"], wide["X"], T, U, V, of, base=base_x, EX=EX, **c.kw())
    for got, ref in zip((Y, T, EX, GU, GV), want):
        assert torch.equal(got, ref)
    for buf, cols in ((oy, c.n), (ox, c.m)):
        buf[1:b + 1, 16:16 + cols] = 7.0
        assert (buf == 7.0).all()
    # the base's own buffer takes the result
    binding.halo_adapters_fwd(wide["X"], U, V, of, base=base_y, Y=base_y, **c.kw())
    binding.halo_adapters_bwd(wide["E"], wide["X"], T, U, V, of, base=base_x, EX=base_x, **c.kw())
    assert torch.equal(base_y, want[0]) and torch.equal(base_x, want[2])


def test_unaligned_index_vectors():
    """adapter_of, ranks and scale are 4-byte aligned only."""
    c = Case(37, 64, 64, 3, 8, scattered(37, 3), ranks=[8, 3, 5])
    want = c.run()
    shift = lambda a: torch.cat([torch.zeros(1, dtype=a.dtype, device=a.device), a])[1:]
    X, E, U, V = (gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V))
    kw = c.kw()
    kw["ranks"], kw["scale"], of = shift(kw["ranks"]), shift(kw["scale"]), shift(gu.to_dev(c.of))
    assert of.data_ptr() % 16 == 4
    Y, T = binding.halo_adapters_fwd(X, U, V, of, base=c.dev_base(c.base_y), **kw)
    got = (Y, T) + binding.halo_adapters_bwd(E, X, T, U, V, of, base=c.dev_base(c.base_x), **kw)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("want", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1), (1, 0, 1)])
def test_gradients_that_are_not_wanted(want):
    c = Case(150, 136, 264, 3, 32, runs(150, 3, 20), p=0.1)
    full = c.run()
    X, E, U, V, T = *(gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V)), full[1]
    got = binding.halo_adapters_bwd(E, X if want[1] else None, T if want[2] else None, U, V, gu.to_dev(c.of),
                                    base=c.dev_base(c.base_x), want_ex=bool(want[0]), want_gu=bool(want[1]), want_gv=bool(want[2]), **c.kw())
    for g, w, ref in zip(got, want, full[2:]):
        assert (g is None) == (not w) and (g is None or torch.equal(g, ref))


def test_no_tokens():
    c = Case(0, 64, 72, 3, 8, [])
    GU, GV = (torch.full(a.shape, 3.0, device=gu.DEV) for a in (c.U, c.V))
    X, E, U, V = (gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V))
    of, T = gu.to_dev(c.of), torch.empty((0, 8), device=gu.DEV)
    Y, _ = binding.halo_adapters_fwd(X, U, V, of, **c.kw())
    EX, _, _ = binding.halo_adapters_bwd(E, X, T, U, V, of, GU=GU, GV=GV, **c.kw())
    torch.cuda.synchronize()
    assert Y.shape == (0, 72) and EX.shape == (0, 64) and not GU.any() and not GV.any()


@pytest.mark.parametrize("b,rank", [(5, 16), (300, 64), (3000, 24)])
def test_same_inputs_same_bits_on_any_stream(b, rank):
    c = Case(b, 264, 520, 6, rank, scattered(b, 6), p=0.1)
    want = c.run()
    for stream in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            got = c.run()
        for a, b_ in zip(got, want):
            assert torch.equal(a, b_)


def test_replays_of_a_graph():
    """Captured once, replayed with other inputs between the program's own work."""
    c = Case(200, 264, 328, 5, 16, scattered(200, 5), p=0.1)
    X, E, U, V, of = *(gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V)), gu.to_dev(c.of)
    base_y, base_x, kw = c.dev_base(c.base_y), c.dev_base(c.base_x), c.kw()
    def step():
        Y, T = binding.halo_adapters_fwd(X, U, V, of, base=base_y, **kw)
        Z = binding.halo_dropout(Y, 0.5, 11, 12)
        return (Y, T, Z) + binding.halo_adapters_bwd(E, X, T, U, V, of, base=base_x, **kw)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(4):
        X.copy_(torch.randn(X.shape, device=gu.DEV)); E.copy_(torch.randn(E.shape, device=gu.DEV))
        of.copy_(torch.randint(-1, 5, of.shape, device=gu.DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), k


def test_offsets_beyond_32_bits():
    """Pools and rows whose elements lie more than 2^32 bytes, and 2^31 elements, from the first."""
    slots, rank, m, n = 300, 128, 65536, 64                    # U: 2.5e9 elements
    U = torch.zeros((slots, rank, m), dtype=torch.bfloat16, device=gu.DEV)
    V = torch.zeros((slots, n, rank), dtype=torch.bfloat16, device=gu.DEV)
    g = torch.Generator(device=gu.DEV).manual_seed(1)
    last = slots - 1
    U[last] = torch.randn((rank, m), generator=g, device=gu.DEV) * m ** -0.5
    V[last] = torch.randn((n, rank), generator=g, device=gu.DEV)
    pitch = 1 << 27                                            # 40 rows of X: 5.4e9 elements
    room = torch.zeros((39 * pitch + m,), dtype=torch.bfloat16, device=gu.DEV)
    X = torch.as_strided(room, (40, m), (pitch, 1))
    X[-4:] = torch.randn((4, m), generator=g, device=gu.DEV)
    of = torch.full((40,), -1, dtype=torch.int32, device=gu.DEV)
    of[-4:] = last
    Y, T = binding.halo_adapters_fwd(X, U, V, of, out_dtype=torch.float32)
    t = X[-4:].double() @ U[last].double().t()
    y = t @ V[last].double().t()
    assert (T[-4:].double() - t).norm() <= 1e-5 * t.norm() and (Y[-4:].double() - y).norm() <= 1e-5 * y.norm()
    assert not Y[:-4].any()
    E = torch.zeros((40, n), dtype=torch.bfloat16, device=gu.DEV)
    E[-4:] = torch.randn((4, n), generator=g, device=gu.DEV)
    EX, GU, GV = binding.halo_adapters_bwd(E, X, T, U, V, of, out_dtype=torch.float32)
    s = E[-4:].double() @ V[last].double()
    ex, gu_, gv = s @ U[last].double(), s.t() @ X[-4:].double(), E[-4:].double().t() @ T[-4:].double()
    for got, want in ((EX[-4:], ex), (GU[last], gu_), (GV[last], gv)):
        assert (got.double() - want).norm() <= 1e-5 * want.norm()
    assert not GU[0].any() and not EX[:-4].any()


@pytest.mark.parametrize("p", [0.0, 0.25])
def test_gradients_against_differences(p):
    """L = <E, Y> is linear in each of X, U and V: the difference of two forward passes is the gradient times the step."""
    c = Case(90, 200, 136, 3, 16, scattered(90, 3), p=p, base=False)
    _, T, EX, GU, GV = c.run()
    X, E, U, V, of = *(gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V)), gu.to_dev(c.of)
    loss = lambda X, U, V: (binding.halo_adapters_fwd(X, U, V, of, **c.kw())[0].double() * E.double()).sum()
    other = lambda t: torch.randn(t.shape, device=gu.DEV).mul_(t.float().std()).to(torch.bfloat16)
    for k, grad in ((0, EX), (1, GU), (2, GV)):
        args = [X, U, V]
        before = loss(*args)
        moved = other(args[k])
        step = moved.double() - args[k].double()
        args[k] = moved
        diff, want = loss(*args) - before, (grad.double() * step).sum()
        # two losses, each a sum of fp32 values with relative errors below (80 + 200/8 + 16) u of the sum of absolute terms
        size = sum((binding.halo_adapters_fwd(a.abs(), b.abs(), v.abs(), of, **dict(c.kw(), scale=c.kw()["scale"].abs()))[0].double()
                    * E.abs().double()).sum() for a, b, v in ((X, U, V), args))
        assert abs(diff - want) <= 2 * (80 + 25 + 16) * U32 * size, (k, float(diff), float(want))


def test_refusals_of_the_binding():
    c = Case(20, 64, 72, 2, 8, scattered(20, 2))
    X, E, U, V, of = *(gu.bits_to_dev(a) for a in (c.X, c.E, c.U, c.V)), gu.to_dev(c.of)
    f = lambda *a, **k: binding.halo_adapters_fwd(*a, **k)
    for bad in ((X.float(), U, V, of), (X[:, :32], U, V, of), (X, U, V.float(), of), (X, U[:1], V, of), (X, U, V, of.long()), (X, U, V, of[:-1]),
                (X.t(), U, V, of), (X, U[:, :, ::2], V, of)):
        with pytest.raises(AssertionError):
            f(*bad)
    with pytest.raises(ValueError):
        f(X.cpu(), U, V, of)
    for kw in (dict(base=X), dict(base=torch.zeros(20, 72, device=gu.DEV)), dict(ranks=torch.zeros(3, dtype=torch.int32, device=gu.DEV)),
               dict(scale=torch.zeros(2, dtype=torch.float64, device=gu.DEV)), dict(T=torch.zeros(20, 16, device=gu.DEV)),
               dict(Y=torch.zeros(72, 20, dtype=torch.bfloat16, device=gu.DEV).t())):
        with pytest.raises(AssertionError):
            f(X, U, V, of, **kw)
    with pytest.raises(binding.HaloError) as e:
        f(X, U, V, of, dropout_p=1.5)
    assert e.value.status == binding.HALO_EINVAL
    with pytest.raises((OverflowError, TypeError)):
        f(X, U, V, of, seed=-1)
    with pytest.raises(binding.HaloError) as e:
        binding.halo_adapters_bwd(E, None, None, U, V, of)
    assert e.value.status == binding.HALO_EINVAL
    with pytest.raises(binding.HaloError) as e:
        f(torch.zeros(20, 65, dtype=torch.bfloat16, device=gu.DEV)[:, 1:], U, V, of)
    assert e.value.status == binding.HALO_EALIGN
