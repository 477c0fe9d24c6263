"""GPU: halo_adapters_* where the kernel of Y and E_X takes tiles of 64, 128 and 256 tokens, against 64-bit torch on the same inputs, with
the bounds of the tests at small sizes (test_gpu_adapters.py).  The mask is halo_dropout's, which has tests of its own.

Requests begin and end inside tiles, some tokens name no adapter, the last ones change it from token to token; adapters have ranks of
their own; what is not used (beyond the ranks, an adapter without tokens, the rows of tokens without one) is NaN."""
import pytest
import torch

from paper_2501_02625_amd import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
SLOTS, NARROW = 5, 72                # adapters, of which the last has no tokens; the width that is not the result's
# rank, tokens, columns of the result, tokens of a tile
SHAPES = [(16, 4097, 7688, 256), (8, 1030, 15880, 64), (16, 200, 65544, 64), (16, 250, 131080, 256), (24, 2055, 16392, 256),
          (32, 1030, 16392, 64), (64, 4097, 7688, 256), (48, 1030, 15880, 64), (56, 130, 98312, 64), (72, 2055, 7688, 128),
          (128, 2055, 7688, 128)]
# type, p, base
FORMS = [(torch.float32, 0.0, "given"), (torch.bfloat16, 0.2, "in place"), (torch.float32, 0.2, "none"), (torch.bfloat16, 0.0, "none")]


class Inputs:
    def __init__(self, rank, b, m, n, p, odt, seed):
        g = torch.Generator(device=gu.DEV).manual_seed(seed)
        normal = lambda *shape, std=1.0: (torch.randn(shape, generator=g, device=gu.DEV) * std).to(torch.bfloat16)
        self.b, self.m, self.n, self.rank, self.p, self.odt, self.seed, self.offset = b, m, n, rank, p, odt, 2**62 + seed, 2**35 + b
        self.X, self.E = normal(b, m), normal(b, n, std=0.5)
        self.U, self.V = normal(SLOTS, rank, m, std=m ** -0.5), normal(SLOTS, n, rank, std=0.3)
        self.T = torch.randn((b, rank), generator=g, device=gu.DEV)
        self.scale = torch.randn(SLOTS, generator=g, device=gu.DEV) + 1.5
        self.ranks = torch.tensor([rank, 1, rank - 3, (rank + 1) // 2, rank], dtype=torch.int32, device=gu.DEV)
        length = max(3, b // 11)
        of = (torch.arange(b, device=gu.DEV) + 17) // length % SLOTS
        of[-b // 8:] = torch.randint(-1, SLOTS - 1, (len(of[-b // 8:]),), generator=g, device=gu.DEV)
        of[of == SLOTS - 1] = -1
        self.of = of.to(torch.int32)
        nan = float("nan")
        self.U[-1], self.V[-1] = nan, nan
        for a, r in enumerate(self.ranks.tolist()):
            self.U[a, r:], self.V[a, :, r:] = nan, nan
        self.X[of < 0], self.E[of < 0] = nan, nan
        self.kw = dict(ranks=self.ranks, scale=self.scale, dropout_p=p, seed=self.seed, offset=self.offset, out_dtype=odt)

    def adapters(self):
        for a, r in enumerate(self.ranks.tolist()):
            t = (self.of == a).nonzero()[:, 0]
            if len(t):
                yield a, r, t, self.U[a, :r].double(), self.V[a, :, :r].double(), self.scale[a].double()

    def factors(self):
        """What drop() multiplies each element of X by, in 64 bits; None: 1."""
        if not self.p:
            return None
        keep = binding.halo_dropout(torch.ones((self.b, self.m), device=gu.DEV), self.p, self.seed, self.offset) != 0
        return keep.double() * (65536.0 / (65536 - round(65536 * self.p)))

    def base(self, cols, form):
        """Base, where the result goes, and the buffer that holds it: the result lies between columns that stay as they are."""
        g = torch.Generator(device=gu.DEV).manual_seed(cols)
        room = torch.full((self.b + 2, cols + 32), 7.0, dtype=self.odt, device=gu.DEV)
        out = room[1:self.b + 1, 16:16 + cols]
        base = None if form == "none" else torch.randn((self.b, cols), generator=g, device=gu.DEV).to(self.odt)
        if form == "in place":
            out.copy_(base)
        return base, (out if form == "in place" else base), out, room

    def out_bound(self, y):
        return (4 * U32 + (2.0 ** -8 if self.odt == torch.bfloat16 else 0.0)) * y.abs()


def within(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d outside the bound; first at %s: got %r want %r bound %r"
                             % (what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(bound[i])))


def untouched(room, out):
    out.fill_(7.0)
    return bool((room == 7.0).all())


@pytest.mark.parametrize("rank,b,wide,tile", SHAPES)
@pytest.mark.parametrize("odt,p,form", FORMS)
def test_forward(rank, b, wide, tile, odt, p, form):
    c = Inputs(rank, b, NARROW, wide, p, odt, seed=rank + b)
    base, given, out, room = c.base(wide, form)
    Y, T = binding.halo_adapters_fwd(c.X, c.U, c.V, c.of, base=given, Y=out, **c.kw)
    again = Y.clone()
    if form == "in place":
        out.copy_(base)
    assert torch.equal(binding.halo_adapters_fwd(c.X, c.U, c.V, c.of, base=given, Y=out, **c.kw)[0], again)
    f = c.factors()
    y = torch.zeros((b, wide), dtype=torch.float64, device=gu.DEV) if base is None else base.double()
    t, ay, at = torch.zeros((b, rank), dtype=torch.float64, device=gu.DEV), torch.zeros_like(y), torch.zeros((b, rank), dtype=torch.float64, device=gu.DEV)
    for a, r, mine, U, V, s in c.adapters():
        x = c.X[mine].double() * (1.0 if f is None else f[mine])
        t[mine, :r], at[mine, :r] = x @ U.t(), x.abs() @ U.abs().t()
        y[mine] += s * (t[mine, :r] @ V.t())
        ay[mine] = s.abs() * (at[mine, :r] @ V.abs().t())
    within(T, t, (40 + NARROW / 8) * U32 * at, "T")
    within(Y, y, ((40 + NARROW / 8) + (40 + rank)) * U32 * ay + c.out_bound(y), "Y")
    assert untouched(room, out)


@pytest.mark.parametrize("rank,b,wide,tile", SHAPES)
@pytest.mark.parametrize("odt,p,form", FORMS)
def test_backward(rank, b, wide, tile, odt, p, form):
    c = Inputs(rank, b, wide, NARROW, p, odt, seed=rank + b)
    base, given, out, room = c.base(wide, form)
    EX, GU, GV = binding.halo_adapters_bwd(c.E, c.X, c.T, c.U, c.V, c.of, base=given, EX=out, **c.kw)
    kept = EX.clone(), GU, GV
    if form == "in place":
        out.copy_(base)
    for x, z in zip(binding.halo_adapters_bwd(c.E, c.X, c.T, c.U, c.V, c.of, base=given, EX=out, **c.kw), kept):
        assert torch.equal(x, z)
    f = c.factors()
    ex = torch.zeros((b, wide), dtype=torch.float64, device=gu.DEV) if base is None else base.double()
    aex = torch.zeros_like(ex)
    want = {a: (0.0, 0.0, 0.0, 0.0, 0) for a in range(SLOTS)}
    for a, r, mine, U, V, s in c.adapters():
        e, t = c.E[mine].double(), c.T[mine, :r].double()
        ff = 1.0 if f is None else f[mine]
        x = torch.where(f[mine] == 0, 0.0, c.X[mine].double() * ff) if f is not None else c.X[mine].double()
        small, asmall = s * (e @ V), s.abs() * (e.abs() @ V.abs())
        ex[mine] += (small @ U) * ff
        aex[mine] = (asmall @ U.abs()) * ff
        want[a] = (small.t() @ x, asmall.t() @ x.abs(), s * (e.t() @ t), s.abs() * (e.abs().t() @ t.abs()), r)
    within(EX, ex, ((40 + NARROW / 8) + (40 + rank)) * U32 * aex + c.out_bound(ex), "EX")
    for a, (gu_, agu, gv, agv, r) in want.items():
        assert not GU[a, r:].any() and not GV[a, :, r:].any()
        if r:
            within(GU[a, :r], gu_, ((40 + NARROW / 8) + (40 + b / 8)) * U32 * agu, "GU")
            within(GV[a, :, :r], gv, (40 + b / 8) * U32 * agv, "GV")
    assert untouched(room, out)
