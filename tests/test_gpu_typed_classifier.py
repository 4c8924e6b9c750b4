"""The example that runs the grouped products, their gradients, AdamW and the 8-bit products together: a typed classifier trained on
the 8-bit multiplier, served on a larger one."""
import os
import sys

import pytest
import torch

from util import ensure_built

pytestmark = pytest.mark.gpu

ensure_built()
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import typed_classifier as T  # noqa: E402


@pytest.mark.parametrize("states", [32, 8])
def test_trains_and_serves(states):
    small, big = T.Multiplier(8), T.Multiplier(32, transposed=False)
    model = T.TypedClassifier(small.X.shape[1])
    first, last = T.train(model, small, 300, states=states)
    assert last < 0.5 * first, (first, last)
    with torch.no_grad():
        full, served = model(big), T.Served(model)(big)
    assert T.accuracy(full, big) > 0.9
    assert T.accuracy(served, big) > T.accuracy(full, big) - 0.05


def test_typed_layer_gradients_against_autograd():
    """the typed layer's autograd function against torch on weights picked row by row, in 64 bits"""
    m = T.Multiplier(8)
    n, K, N = m.X.shape[0], 12, 20
    gen = torch.Generator(device="cuda").manual_seed(1)
    X, W, b = (torch.randn(s, generator=gen, device="cuda").requires_grad_(True) for s in ((n, K), (3, K, N), (3, N)))
    R = torch.randn((n, N), generator=gen, device="cuda")
    got = torch.autograd.grad((T.Typed.apply(X, W, b, m.offsets) * R).sum(), (X, W, b))
    X64, W64, b64 = (t.detach().cpu().double().requires_grad_(True) for t in (X, W, b))
    of = torch.repeat_interleave(torch.arange(3), torch.diff(m.offsets.cpu()))
    Y = torch.stack([X64[i] @ W64[of[i]] + b64[of[i]] for i in range(n)])
    want = torch.autograd.grad((Y * R.cpu().double()).sum(), (X64, W64, b64))
    # sums of N products, of up to n products, of up to n values, every addition and product off by 2^-23 of a partial sum at most
    terms = [R.cpu().double().abs() @ W64.detach().abs().sum(0).t(), X64.detach().abs().t() @ R.cpu().double().abs(), R.cpu().double().abs().sum(0)]
    for g, w, t, adds in zip(got, want, terms, (N, n, n)):
        assert ((g.cpu().double() - w).abs() <= (adds + 3) * 2.0 ** -23 * t).all()


def test_second_derivatives_are_refused():
    """the gradient calls have no gradients of their own: a second derivative would leave out what goes through them"""
    m = T.Multiplier(8)
    X = torch.randn((m.X.shape[0], 12), device="cuda").requires_grad_(True)
    W, b = torch.randn((3, 12, 20), device="cuda").requires_grad_(True), torch.zeros((3, 20), device="cuda")
    for out in (T.Typed.apply(X, W, b, m.offsets), T.Aggregate.apply(X, m)):
        g, = torch.autograd.grad(out.square().sum(), X, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (g * X).sum().backward()


def test_only_the_gradients_that_are_asked_for():
    m = T.Multiplier(8)
    wants = torch.randn((m.X.shape[0], 12), device="cuda"), torch.randn((3, 12, 20), device="cuda"), torch.randn((3, 20), device="cuda")
    R = torch.randn((m.X.shape[0], 20), device="cuda")
    full = torch.autograd.grad((T.Typed.apply(*(t.requires_grad_(True) for t in wants), m.offsets) * R).sum(), wants)
    for ask in ((0,), (1,), (2,), (0, 2), (1, 2)):
        some = [t.detach().requires_grad_(i in ask) for i, t in enumerate(wants)]
        got = torch.autograd.grad((T.Typed.apply(*some, m.offsets) * R).sum(), [some[i] for i in ask])
        assert all(torch.equal(g, full[i]) for g, i in zip(got, ask))
