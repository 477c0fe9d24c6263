"""GPU: the example's layer takes each training pass's gradients with the masks of that pass, whatever passes ran in between."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
TOKENS, WIDTH, SLOTS, RANK, P = 96, 256, 3, 8, 0.5      # the factor of p = 0.5 is 2: no rounding


@pytest.fixture(scope="module")
def layer():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "many_adapters.py")
    spec = importlib.util.spec_from_file_location("many_adapters", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    g = torch.Generator(device="cuda").manual_seed(1)
    layer = example.Layer((torch.randn((WIDTH, WIDTH), generator=g, device="cuda") * WIDTH ** -0.5).to(torch.bfloat16), SLOTS, RANK, P, 5)
    layer.V = torch.randn((SLOTS, WIDTH, RANK), generator=g, device="cuda")
    return layer


def inputs(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    X, E = (torch.randn((TOKENS, WIDTH), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    return X, E, (torch.arange(TOKENS, device="cuda") * 7 % SLOTS).to(torch.int32)


def check(layer, X, E, of, out_mask, T, grads, factor):
    """G_V = E_masked^T T; and <G_U, U> = sum of S_t T_t = <G_V, V> for every adapter, if G_U has the mask that T was made with.
    out_mask: of the residual branch, or None.  Bounds: fp32 sums with at most one rounding per eight products, as in the kernels' tests."""
    _, GU, GV = (t.double() for t in grads)
    U, V = (t.double() for t in layer.adapters())
    e = E.double() if out_mask is None else torch.where(out_mask, E.double() * 2, 0.0)
    for a in range(SLOTS):
        t = (of == a).nonzero()[:, 0]
        want, size = e[t].t() @ T[t].double(), e[t].abs().t() @ T[t].double().abs()
        assert ((GV[a] - want).abs() <= (40 + TOKENS / 8) * U32 * size).all()
        terms = ((e[t].abs() @ V[a].abs()) * (X[t].double().abs() @ U[a].abs().t()) * factor).sum()
        assert abs((GU[a] * U[a]).sum() - (GV[a] * V[a]).sum()) <= (160 + (2 * WIDTH + WIDTH + 2 * TOKENS) / 8) * U32 * terms


@pytest.mark.parametrize("order", [(0, 1, 2), (2, 0, 1)])
def test_passes_whose_gradients_are_taken_later(layer, order):
    passes = []
    for k in range(3):
        X, E, of = inputs(k if k < 2 else 0)
        out, saved = layer.forward(X, of, residual=torch.zeros_like(X), train=True)
        passes.append((X, E, of, out, saved))
    masks = [q[3] != 0 for q in passes]
    assert not torch.equal(masks[0], masks[2]) and not torch.equal(passes[0][4][1], passes[2][4][1])      # the same X
    for k in order:
        X, E, of, out, saved = passes[k]
        check(layer, X, E, of, masks[k], saved[1], layer.backward(E, saved), 2.0)


def test_without_a_residual_no_mask_is_on_the_result(layer):
    X, E, of = inputs(7)
    _, saved = layer.forward(X, of, train=True)
    check(layer, X, E, of, None, saved[1], layer.backward(E, saved), 2.0)


def test_a_pass_without_dropout(layer):
    X, E, of = inputs(8)
    _, saved = layer.forward(X, of, residual=torch.zeros_like(X))
    check(layer, X, E, of, None, saved[1], layer.backward(E, saved), 1.0)
