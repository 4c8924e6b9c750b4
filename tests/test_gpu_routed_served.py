"""The served form of the routed example, call by call: what goes into every call is what the calls before it gave, and what comes out is the layer's
formula in 64 bits on that input.

u = 2^-24.  A sum of K products in fp32 is within (K + 2) 2 u of its terms' magnitudes.  A value cut to 8 bits is off by half a step, the row's scale, and by the
rounding of a quotient of at most 127: 0.5 + 2^-16 steps.  An 8-bit product is exact up to three roundings of fp32: 4 u of its terms.
"""
import os
import sys

import pytest
import torch

from util import ensure_built

pytestmark = pytest.mark.gpu

ensure_built()
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paper_2511_18297_amd as G  # noqa: E402
import routed_classifier as R  # noqa: E402

U, HALF = 2.0 ** -24, 0.5 + 2.0 ** -16
CALLS = ["groot_spmm_execute", "groot_grouped_product", "groot_rms_norm", "groot_grouped_product", "groot_route", "groot_routed_rows", "groot_quantized_product",
         "groot_quantized_linear", "groot_routed_sum"]


class Call:
    """a call's tensors as they were before it and after it"""

    def __init__(self, name, args, more, run):
        def copies(x):
            return x.clone() if isinstance(x, torch.Tensor) else x
        self.name, self.before = name, [copies(a) for a in args]
        run(*args, **more)
        self.after, self.named = [copies(a) for a in args], {k: copies(v) for k, v in more.items()}


def near(got, want, terms, per, what):
    err = (got.double() - want).abs()
    assert bool((err <= per * terms + 1e-38).all()), f"{what}: {float((err / (per * terms + 1e-38)).max())} of the tolerance"


def product(x, w, bias):
    """x w + bias in 64 bits, and its terms' magnitudes"""
    x, w = x.double(), w.detach().double()
    b = 0 if bias is None else bias.detach().double()
    return x @ w + b, x.abs() @ w.abs() + (0 if bias is None else b.abs())


def cut_is_near(Q, scale, x, what):
    err = (Q.double() * scale.double()[..., None] - x.double()).abs()
    assert bool((err <= HALF * scale.double()[..., None]).all()), what


def test_every_call_of_the_served_layers(monkeypatch):
    m = R.Multiplier(8, transposed=False)
    gen = torch.Generator(device="cuda").manual_seed(500)
    model = R.RoutedClassifier(m.X.shape[1])
    with torch.no_grad():                                   # nothing is at its first value
        for p in model.parameters():
            p += 0.1 * torch.randn(p.shape, generator=gen, device="cuda")
        model.bias = [0.05 * torch.randn(R.EXPERTS, generator=gen, device="cuda") for _ in model.bias]
    served, calls = R.ServedRouted(model), []
    for name in set(CALLS):
        def record(*args, run=getattr(G, name), name=name, **more):
            calls.append(Call(name, args, more, run))
        monkeypatch.setattr(G, name, record)
    with torch.no_grad():
        logits = served(m)
    monkeypatch.undo()
    assert [c.name for c in calls] == ["groot_grouped_product"] + CALLS * len(model.layers) + ["groot_grouped_product"]
    view = G.groot_graph_view(m.graph)
    n = m.X.shape[0]
    A = torch.sparse_csr_tensor(*(torch.from_numpy(view[k].copy()) for k in ("rowptr", "col")), torch.from_numpy(view["val"].copy()).double(), size=(n, n)).to_dense().cuda()

    first, last = calls[0], calls[-1]
    assert torch.equal(first.before[0], m.X)
    near(first.after[5], *product(m.X, model.inp[0][0], model.inp[1][0]), (m.X.shape[1] + 2) * 2 * U, "input layer")
    h = first.after[5]
    for i, p in enumerate(model.layers):
        spmm, own, norm, score, route, rows, up, down, total = calls[1 + 9 * i:10 + 9 * i]
        assert torch.equal(spmm.before[1], h) and torch.equal(own.before[0], spmm.after[2])
        near(spmm.after[2], A @ h.double(), A.abs() @ h.double().abs(), (n + 2) * 2 * U, "aggregation")
        near(own.after[5], *product(own.before[0], p["Wa"][0], None), (R.WIDTH + 2) * 2 * U, "aggregated features")

        x, residual, gain = norm.before[:3]
        y, held, Q, q_scale = norm.after[4], norm.named["H"], norm.named["Q"], norm.named["q_scale"]
        assert torch.equal(x, own.after[5]) and torch.equal(residual, h) and torch.equal(gain, p["gain"]) and torch.equal(held, x + residual)
        want = held.double() / torch.sqrt(held.double().square().mean(1, keepdim=True) + R.EPS) * gain.double()
        near(y, want, want.abs(), 4.1 * U, "norm")
        cut_is_near(Q, q_scale, y, "norm in 8 bits")
        h = held

        assert torch.equal(score.before[0], y)
        near(score.after[5], *product(y, p["Wr"][0], None), (R.WIDTH + 2) * 2 * U, "scores")
        scores, bias = route.before[:2]
        chosen, weights, places, offsets = route.after[2:6]
        assert torch.equal(scores, score.after[5]) and torch.equal(bias, model.bias[i])
        gates = torch.sigmoid(scores.double())
        assert torch.equal(chosen.long(), torch.topk(gates + bias.double(), R.CHOSEN, dim=1).indices)
        w = torch.gather(gates, 1, chosen.long())
        w = w / w.sum(1, keepdim=True)
        near(weights, w, w, (float(scores.abs().max()) + 40) * 2 * U, "weights")
        order = torch.sort(chosen.reshape(-1).long(), stable=True).indices
        assert torch.equal(places.reshape(-1)[order].long(), torch.arange(n * R.CHOSEN, device="cuda"))
        assert torch.equal(torch.diff(offsets), torch.bincount(chosen.reshape(-1).long(), minlength=R.EXPERTS))

        R8, r_scale = rows.after[2], rows.after[4]
        assert torch.equal(rows.before[0], Q) and torch.equal(rows.before[1], places) and torch.equal(rows.before[3], q_scale)
        at, of = places.reshape(-1).long(), torch.arange(n, device="cuda").repeat_interleave(R.CHOSEN)
        assert torch.equal(R8[at], Q[of]) and torch.equal(r_scale[at], q_scale[of])

        V8, v_scale, U8, u_scale = up.before[2], up.before[3], down.before[1], down.before[2]
        cut_is_near(V8, v_scale, p["V"].detach().transpose(1, 2), "V")
        cut_is_near(U8, u_scale, p["U"].detach().transpose(1, 2), "U")
        assert torch.equal(up.before[0], R8) and torch.equal(up.before[1], r_scale) and torch.equal(up.before[4], offsets) and torch.equal(up.before[5], p["c"])
        inner = up.after[7]
        assert torch.equal(down.before[0], inner) and torch.equal(down.before[3], offsets)
        answer = down.after[6]
        for e in range(R.EXPERTS):
            r = slice(int(offsets[e]), int(offsets[e + 1]))
            exact, terms = product(R8[r].double() * r_scale[r, None].double(), (V8[e].double() * v_scale[e, :, None].double()).t(), p["c"][e])
            near(inner[r], torch.relu(exact), terms, 4 * U, "experts' first product")
            weight = U8[e].double() * u_scale[e, :, None].double()
            exact, terms = product(inner[r], weight.t(), None)
            step = inner[r].double().abs().amax(1, keepdim=True) / 127 * (1 + 4 * U)
            assert bool(((answer[r].double() - exact).abs() <= HALF * step * weight.abs().sum(1) + 8 * U * terms + 1e-38).all()), "experts' second product"

        assert torch.equal(total.before[0], answer) and torch.equal(total.before[1], places) and torch.equal(total.before[2], weights) and torch.equal(total.before[3], h)
        parts = answer.double()[places.long()] * weights.double()[:, :, None]
        near(total.after[4], h.double() + parts.sum(1), h.double().abs() + parts.abs().sum(1), (R.CHOSEN + 2) * 2 * U, "the experts' answers in the stream")
        h = total.after[4]
    assert torch.equal(last.before[0], h) and torch.equal(last.after[5], logits)
    near(logits, *product(h, model.out[0][0], model.out[1][0]), (R.WIDTH + 2) * 2 * U, "logits")
