"""The example that runs the routing calls, the norm, the grouped products and the 8-bit products together."""
import os
import subprocess
import sys

import pytest
import torch

from util import ensure_built

pytestmark = pytest.mark.gpu

ensure_built()
EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
sys.path.insert(0, EXAMPLES)
import paper_2511_18297_amd as G  # noqa: E402
import routed_classifier as R  # noqa: E402


def test_trains_and_serves():
    """it runs: losses, logits and the experts' shares are finite and whole"""
    small, big = R.Multiplier(8), R.Multiplier(16, transposed=False)
    model = R.RoutedClassifier(small.X.shape[1])
    first, last = R.train(model, small, 20)
    assert first == first and last == last
    assert all(int(o[-1]) == small.X.shape[0] * R.CHOSEN for o in model.offsets)
    with torch.no_grad():
        full, served = model(big), R.ServedRouted(model)(big)
    assert torch.isfinite(full).all() and torch.isfinite(served).all() and full.shape == served.shape


def test_the_command_runs():
    out = subprocess.run([sys.executable, os.path.join(EXAMPLES, "routed_classifier.py"), "--infer-bits", "16", "--epochs", "3"], capture_output=True, text=True,
                         timeout=110)
    assert out.returncode == 0 and "accuracy" in out.stdout, out.stderr


def reference(model, m, rows):
    """the model in 64 bits on the CPU, and its parameters"""
    p = [t.detach().cpu().double().requires_grad_(True) for t in model.parameters()]
    (W, b), (Wo, bo), rest = p[0:2], p[2:4], p[4:]
    rowptr, col, val = rows
    n = len(rowptr) - 1
    A = torch.sparse_csr_tensor(torch.from_numpy(rowptr.copy()), torch.from_numpy(col.copy()).long(), torch.from_numpy(val.copy()).double(), size=(n, n)).to_dense()
    h = m.X.cpu().double() @ W[0] + b[0]
    for i in range(len(model.layers)):
        Wa, gain, Wr, V, c, U = rest[6 * i:6 * i + 6]
        h = h + (A @ h) @ Wa[0]
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + R.EPS) * gain
        score = torch.sigmoid(y @ Wr[0])
        experts = torch.topk(score + model.bias[i].cpu().double(), R.CHOSEN, dim=1).indices
        w = torch.gather(score, 1, experts)
        w = w / w.sum(1, keepdim=True)
        every = torch.relu(torch.einsum("nk,ekj->nej", y, V) + c)
        answers = torch.einsum("nej,ejk->nek", every, U)
        h = h + (torch.gather(answers, 1, experts[:, :, None].expand(-1, -1, R.WIDTH)) * w[:, :, None]).sum(1)
    return h @ Wo[0] + bo[0], p


def test_gradients_of_the_whole_model():
    """Every parameter's gradient against autograd in 64 bits.  Sums of up to 960 products in fp32 lose 960 x 2^-23 = 2^-13 of their terms' magnitudes at the
    most, and a path from the loss to a parameter has ten of them: 2^-10 of the largest gradient's magnitude."""
    m = R.Multiplier(8)
    model = R.RoutedClassifier(m.X.shape[1])
    model.bias = [torch.randn(R.EXPERTS, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 0.05 for _ in model.bias]
    view = G.groot_graph_view(m.graph)
    along = torch.randn((m.X.shape[0], R.CLASSES), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    got = torch.autograd.grad((model(m) * along).sum(), model.parameters())
    out, p = reference(model, m, (view["rowptr"], view["col"], view["val"]))
    want = torch.autograd.grad((out * along.cpu().double()).sum(), p)
    for i, (g, w) in enumerate(zip(got, want)):
        assert g.shape == w.shape and float((g.cpu().double() - w).abs().max()) <= 2.0 ** -10 * float(w.abs().max()), i


def test_second_derivatives_are_refused():
    x, s = (torch.randn((9, 24), device="cuda").requires_grad_(True) for _ in range(2))
    for out in (R.Norm.apply(x, s, torch.ones(24, device="cuda"))[1], R.Route.apply(x, None)[0]):
        g, = torch.autograd.grad(out.square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (g * x).sum().backward()


def test_only_the_gradients_that_are_asked_for():
    gen = torch.Generator(device="cuda").manual_seed(5)
    weights, _, places, _ = R.Route.apply(torch.randn((50, 8), generator=gen, device="cuda"), None)
    rows, stream, along = (torch.randn(s, generator=gen, device="cuda") for s in ((100, 24), (50, 24), (50, 24)))
    wants = [rows.requires_grad_(True), weights.requires_grad_(True), stream.requires_grad_(True)]

    def sums(a, w, b):
        return (R.FromExperts.apply(a, places, w, b) * along).sum()
    full = torch.autograd.grad(sums(*wants), wants)
    for ask in ((0,), (1,), (2,), (0, 2), (1, 2), (0, 1)):
        some = [t.detach().requires_grad_(i in ask) for i, t in enumerate(wants)]
        got = torch.autograd.grad(sums(*some), [some[i] for i in ask])
        assert all(torch.equal(g, full[i]) for g, i in zip(got, ask))
