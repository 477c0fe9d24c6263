"""The operators around a layer's products as a training step runs them, on an MLP block with a residual connection:

    h = norm(x);  a = gelu(h W1^T + b1);  y = a W2^T + b2 + x

forward and backward through halo_layer_norm_*, halo_linear_*_epilogue, halo_activation_bwd, halo_linear_bwd, then halo_adamw over all six
parameters; eagerly, in a captured graph, and on a stream of its own."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as orc
from paper_2501_02625_amd import binding
from tests.around_util import HALF, U, act_bound, column_terms, host, within
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
B, D, F = 96, 256, 512
BF = torch.bfloat16


class Block:
    def __init__(self, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=DEV)
        self.x, self.target = r(B, D).to(BF), r(B, D).to(BF)
        self.params = [(1 + 0.1 * r(D)).to(BF), (0.1 * r(D)).to(BF), (r(F, D) * D ** -0.5).to(BF), (0.1 * r(F)).to(BF),
                       (r(D, F) * F ** -0.5).to(BF), (0.1 * r(D)).to(BF)]
        zeros = lambda dtype, per=1: [torch.zeros(-(-p.numel() // per), dtype=dtype, device=DEV) for p in self.params]
        self.m, self.v = zeros(torch.float8_e4m3fn), zeros(torch.float8_e4m3fn)
        self.ms, self.vs = zeros(torch.float32, 256), zeros(torch.float32, 256)
        self.grads = [torch.zeros(p.shape, device=DEV) for p in self.params]
        self.up, self.down = binding.make_desc(B, D, F, 1, BF), binding.make_desc(B, F, D, 1, BF)
        self.up32, self.down32 = binding.make_desc(B, D, F, 1, torch.float32), binding.make_desc(B, F, D, 1, torch.float32)
        self.step = torch.zeros((), dtype=torch.int64, device=DEV)

    def forward(self):
        w, b, W1, b1, W2, b2 = self.params
        self.h, self.mean, self.rstd = binding.halo_layer_norm_fwd(self.x, w, b)
        self.a, self.s1, self.z = binding.halo_linear_fwd_epilogue(self.up, self.h, W1, bias=b1, activation="gelu", want_z=True)
        self.y, self.s2, _ = binding.halo_linear_fwd_epilogue(self.down, self.a, W2, bias=b2, residual=self.x)
        return self.y

    def backward(self, e):
        w = self.params[0]
        _, g = binding.halo_activation_bwd(e, None, "none", want_ez=False)
        self.grads[5].copy_(g)
        ea, _ = binding.halo_linear_bwd(self.down, e, self.s2, want_g=False)
        binding.halo_linear_bwd(self.down32, e, self.s2, want_ex=False, G=self.grads[4])
        ez, _ = binding.halo_activation_bwd(ea, self.z, "gelu", EZ=ea, GB=self.grads[3])
        eh, _ = binding.halo_linear_bwd(self.up, ez, self.s1, want_g=False)
        binding.halo_linear_bwd(self.up32, ez, self.s1, want_ex=False, G=self.grads[2])
        ex, _, _ = binding.halo_layer_norm_bwd(eh, self.x, self.mean, self.rstd, w, base=e, GW=self.grads[0], GB=self.grads[1])
        return ex

    def update(self):
        binding.halo_adamw(self.params, self.grads, self.m, self.v, step=self.step, lr=2e-3, weight_decay=0.1, m_scales=self.ms, v_scales=self.vs,
                           seed=3)

    def train(self):
        self.step += 1
        y = self.forward()
        ex = self.backward((y - self.target) * 0.01)
        self.update()
        return y, ex

    def state(self):
        return [t.clone() for t in self.params + self.grads + self.ms + self.vs] + [t.view(torch.uint8).clone() for t in self.m + self.v]

    def restore(self, s):
        for t, k in zip(self.params + self.grads + self.ms + self.vs + [t.view(torch.uint8) for t in self.m + self.v], s):
            t.copy_(k)
        self.step.zero_()


def test_forward_and_backward_are_those_of_the_parts():
    """Each part against its formula on the inputs that it was given."""
    k = Block()
    y = k.forward()
    w, b, W1, b1, W2, b2 = k.params
    codes = lambda s: (s.Xq.cpu().numpy(), s.Wq.cpu().numpy(), s.s_x.cpu().numpy(), s.s_w.cpu().numpy())
    for s, bias, act, res, got, z in ((k.s1, b1, "gelu", None, k.a, k.z), (k.s2, b2, "none", k.x, y, None)):
        want, wz = orc.product(*codes(s), host(bias), act, None if res is None else host(res))
        off = 6 * U * (np.abs(wz) + np.abs(wz - host(bias)))
        within(got, want, 1.2 * off + act_bound(wz, want, act, BF) + U * np.abs(want) + HALF[BF] * (np.abs(want) + 1e-6), act)
        if z is not None:
            within(z, wz, off + HALF[BF] * (np.abs(wz) + 1e-6), "Z")
    e = ((y - k.target) * 0.01).to(BF)
    ex = k.backward(e)
    within(k.grads[5], host(e).sum(axis=0), column_terms(B) * U * np.abs(host(e)).sum(axis=0), "gradient of b2")
    # the residual's gradient went round the norm: what is left is the norm's own
    alone, _, _ = binding.halo_layer_norm_bwd(binding.halo_linear_bwd(k.up, binding.halo_activation_bwd(
        binding.halo_linear_bwd(k.down, e, k.s2, want_g=False)[0], k.z, "gelu")[0], k.s1, want_g=False)[0], k.x, k.mean, k.rstd, w)
    # both were rounded to bf16 once, alone before the sum
    want = host(alone) + host(e)
    within(ex, want, HALF[BF] * (np.abs(want) + np.abs(host(alone))) * 1.01 + 1e-9, "EX")


def test_gradients_follow_the_layer_without_quantisation():
    """The block in fp32 through autograd.  INT8 codes are 127 steps for a row's largest value, a row's values up to four times its root mean
    square: each of the products is off by about 4 / 127 / sqrt(12), 1 %, of its size for each of its two operands, and three products
    follow one another: well within 10 % in the mean."""
    k = Block(1)
    y = k.forward()
    e = ((y - k.target) * 0.01).to(BF)
    ex = k.backward(e)
    p = [t.float().cpu().requires_grad_() for t in k.params]
    x = k.x.float().cpu().requires_grad_()
    h = torch.nn.functional.layer_norm(x, (D,), p[0], p[1])
    out = torch.nn.functional.gelu(h @ p[2].t() + p[3]) @ p[4].t() + p[5] + x
    out.backward(e.float().cpu())
    for got, want in [(y, out)] + list(zip(k.grads + [ex], [t.grad for t in p] + [x.grad])):
        got, want = got.float().cpu(), want.detach()
        assert (got - want).norm() <= 0.1 * want.norm()


def test_a_graph_of_the_step_is_the_step():
    """Captured once, replayed with other work between: the same bits as eager steps, step by step."""
    eager, k = Block(2), Block(2)
    first = k.state()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        k.train()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = k.train()
    k.restore(first)
    for step in range(4):
        want = eager.train()
        graph.replay()
        assert torch.randn(1000, device=DEV).sum().item() == pytest.approx(0, abs=1e4)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), step
        assert all(torch.equal(a, b) for a, b in zip(k.state(), eager.state())), step


def test_two_graphs_of_two_blocks():
    """Two captured steps, replayed at once on two streams."""
    blocks, graphs, streams = [Block(3), Block(4)], [], [torch.cuda.Stream() for _ in range(2)]
    wants = [Block(3), Block(4)]
    for k in blocks:
        first = k.state()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            k.train()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            k.train()
        k.restore(first)
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for k, want in zip(blocks, wants):
            want.train()
            assert all(torch.equal(a, b) for a, b in zip(k.state(), want.state()))


def test_on_a_stream_of_its_own():
    want, k = Block(5), Block(5)
    want.train()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        k.train()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(k.state(), want.state()))
