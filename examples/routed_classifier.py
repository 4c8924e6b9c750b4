"""A node classifier whose layers are routed to experts, trained and served through the library.

Every layer adds the aggregated features to a stream of features, norms it, sends each node to two of eight small networks and adds what
they answer, weighted, to the stream:
    h <- h + (A_hat h) Wa;   y = rms_norm(h);   h <- h + sum over the chosen experts e of weight_e (relu(y V_e + c_e) U_e)
The experts are kept busy by a bias on their probabilities, moved after every step by how many nodes each of them has.  Training runs
the routing calls, the grouped products and the norm with their gradients; serving cuts the norm's output to 8 bits as it is made,
and the rows travel to 8-bit experts with their scales.

    python examples/routed_classifier.py --bits 8 --infer-bits 32 --epochs 200
"""
import argparse
import os
import sys

import numpy as np
import torch
from torch.autograd.function import once_differentiable

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for path in (ROOT, os.path.join(ROOT, "examples")):
    if path not in sys.path:
        sys.path.insert(0, path)
import paper_2511_18297_amd as G  # noqa: E402
from typed_classifier import CLASSES, AdamW, Aggregate, Multiplier, Served, Typed, accuracy  # noqa: E402

WIDTH, INNER, EXPERTS, CHOSEN, EPS = 32, 64, 8, 2, 1e-6
GATE = dict(gate=G.GROOT_SIGMOID, renormalise=True)


def empty(*shape, like):
    return torch.empty(shape, dtype=like.dtype, device="cuda")


class Norm(torch.autograd.Function):
    """h = x + residual and rms_norm(h) gain"""

    @staticmethod
    def forward(ctx, x, residual, gain):
        x, residual = x.contiguous(), residual.contiguous()
        h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[0], device="cuda")
        G.groot_rms_norm(x, residual, gain, EPS, y, H=h, rstd=rstd)
        ctx.save_for_backward(h, rstd, gain)
        return h, y

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dy):
        h, rstd, gain = ctx.saved_tensors
        dx, dgain, workspace = torch.empty_like(h), None, None
        if ctx.needs_input_grad[2]:
            dgain = torch.empty_like(gain)
            need = G.groot_rms_norm_backward_workspace(*h.shape, h.dtype)
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        G.groot_rms_norm_backward(h, rstd, gain, dy.contiguous(), dx, dgain, workspace, dH=dh.contiguous())
        return dx, dx, dgain


class Route(torch.autograd.Function):
    """weights, experts, places and offsets of every row's choice; the weights have a gradient"""

    @staticmethod
    def forward(ctx, scores, bias):
        scores = scores.contiguous()
        n, experts = scores.shape
        chosen, places = (torch.empty((n, CHOSEN), dtype=torch.int32, device="cuda") for _ in range(2))
        weights, offsets = torch.empty((n, CHOSEN), device="cuda"), torch.empty(experts + 1, dtype=torch.int64, device="cuda")
        workspace = torch.empty(max(G.groot_route_workspace(n, experts, CHOSEN), 16), dtype=torch.uint8, device="cuda")
        G.groot_route(scores, bias, chosen, weights, places, offsets, workspace, **GATE)
        ctx.save_for_backward(scores, chosen)
        ctx.mark_non_differentiable(chosen, places, offsets)
        return weights, chosen, places, offsets

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights, *_):
        scores, chosen = ctx.saved_tensors
        dscores = torch.empty_like(scores)
        G.groot_route_backward(scores, chosen, dweights.contiguous(), dscores, **GATE)
        return dscores, None


class ToExperts(torch.autograd.Function):
    """R[places[i, s]] = X[i]"""

    @staticmethod
    def forward(ctx, X, places):
        X = X.contiguous()
        R = empty(places.numel(), X.shape[1], like=X)
        G.groot_routed_rows(X, places, R)
        ctx.save_for_backward(places)
        return R

    @staticmethod
    @once_differentiable
    def backward(ctx, dR):
        places, = ctx.saved_tensors
        dX = empty(places.shape[0], dR.shape[1], like=dR)
        G.groot_routed_sum(dR.contiguous(), places, None, None, dX)
        return dX, None


class FromExperts(torch.autograd.Function):
    """stream[i] + sum over s of weights[i, s] R[places[i, s]]"""

    @staticmethod
    def forward(ctx, R, places, weights, stream):
        R, weights, stream = R.contiguous(), weights.contiguous(), stream.contiguous()
        out = torch.empty_like(stream)
        G.groot_routed_sum(R, places, weights, stream, out)
        ctx.save_for_backward(R, places, weights)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        R, places, weights = ctx.saved_tensors
        dout = dout.contiguous()
        dR = torch.empty_like(R) if ctx.needs_input_grad[0] else None
        dweights = torch.empty_like(weights) if ctx.needs_input_grad[2] else None
        if dR is not None or dweights is not None:
            G.groot_routed_sum_backward(dout, R, places, weights, dR, dweights)
        return dR, None, dweights, dout


class RoutedClassifier:
    """Two routed layers between an input and an output product."""

    def __init__(self, features, layers=2, seed=7):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weights(groups, a, b):
            return ((torch.rand((groups, a, b), generator=gen, device="cuda") - 0.5) * (2.0 / np.sqrt(a))).requires_grad_(True)

        def zeros(groups, b):
            return torch.zeros((groups, b), device="cuda", requires_grad=True)
        self.inp, self.out = (weights(1, features, WIDTH), zeros(1, WIDTH)), (weights(1, WIDTH, CLASSES), zeros(1, CLASSES))
        self.layers = [dict(Wa=weights(1, WIDTH, WIDTH), gain=torch.ones(WIDTH, device="cuda", requires_grad=True), Wr=weights(1, WIDTH, EXPERTS),
                            V=weights(EXPERTS, WIDTH, INNER), c=zeros(EXPERTS, INNER), U=weights(EXPERTS, INNER, WIDTH)) for _ in range(layers)]
        self.bias = [torch.zeros(EXPERTS, device="cuda") for _ in range(layers)]
        self.offsets = [None] * layers                       # of the last pass: how many nodes each expert had

    def parameters(self):
        return [*self.inp, *self.out] + [p for layer in self.layers for p in layer.values()]

    def __call__(self, m):
        h = Typed.apply(m.X, *self.inp, None)
        for i, p in enumerate(self.layers):
            h, y = Norm.apply(Typed.apply(Aggregate.apply(h, m), p["Wa"], None, None), h, p["gain"])
            weights, _, places, offsets = Route.apply(Typed.apply(y, p["Wr"], None, None), self.bias[i])
            inner = torch.relu(Typed.apply(ToExperts.apply(y, places), p["V"], p["c"], offsets))
            h = FromExperts.apply(Typed.apply(inner, p["U"], None, offsets), places, weights, h)
            self.offsets[i] = offsets
        return Typed.apply(h, *self.out, None)

    def balance(self, rate):
        """experts with fewer nodes than the average are chosen a little sooner"""
        for bias, offsets in zip(self.bias, self.offsets):
            count = torch.diff(offsets).float()
            bias += rate * torch.sign(count.mean() - count)


def train(model, m, epochs, lr=1e-2, rate=1e-3):
    """(first loss, last loss) of full-graph training with classes weighted by how rare they are."""
    counts = torch.bincount(m.y, minlength=CLASSES).float()
    weight = counts.sum() / (CLASSES * counts.clamp(min=1))
    opt = AdamW(model.parameters(), lr, states=32)
    losses = []
    for _ in range(epochs):
        opt.zero_grad()
        loss = torch.nn.functional.cross_entropy(model(m), m.y, weight=weight)
        loss.backward()
        opt.step()
        model.balance(rate)
        losses.append(loss.detach())
    return float(losses[0]), float(losses[-1])


class ServedRouted:
    """The trained layers with the experts' weights in 8 bits; the rows reach them in 8 bits from the norm on."""

    def __init__(self, model):
        self.model = model
        self.layers = [dict(V=Served.cut(p["V"]), U=Served.cut(p["U"])) for p in model.layers]

    def __call__(self, m):
        h = empty(m.X.shape[0], WIDTH, like=m.X)
        (W, b), (Wo, bo) = self.model.inp, self.model.out
        n = h.shape[0]
        G.groot_grouped_product(m.X, W, None, b, False, h)
        agg, near, y, scores = (empty(n, w, like=h) for w in (WIDTH, WIDTH, WIDTH, EXPERTS))
        Q, q_scale = torch.empty((n, WIDTH), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        R8, r_scale = torch.empty((n * CHOSEN, WIDTH), dtype=torch.int8, device="cuda"), torch.empty(n * CHOSEN, device="cuda")
        inner, answer = empty(n * CHOSEN, INNER, like=h).zero_(), empty(n * CHOSEN, WIDTH, like=h)
        chosen, places = (torch.empty((n, CHOSEN), dtype=torch.int32, device="cuda") for _ in range(2))
        weights, offsets = torch.empty((n, CHOSEN), device="cuda"), torch.empty(EXPERTS + 1, dtype=torch.int64, device="cuda")
        route_work = torch.empty(max(G.groot_route_workspace(n, EXPERTS, CHOSEN), 16), dtype=torch.uint8, device="cuda")
        work = torch.empty(G.groot_quantized_linear_workspace(n * CHOSEN, INNER), dtype=torch.uint8, device="cuda")
        for p, bias, served in zip(self.model.layers, self.model.bias, self.layers):
            G.groot_spmm_execute(m.plan, h, agg)
            G.groot_grouped_product(agg, p["Wa"], None, None, False, near)
            G.groot_rms_norm(near, h, p["gain"], EPS, y, H=h, Q=Q, q_scale=q_scale)          # the stream in place
            G.groot_grouped_product(y, p["Wr"], None, None, False, scores)
            G.groot_route(scores, bias, chosen, weights, places, offsets, route_work, **GATE)
            G.groot_routed_rows(Q, places, R8, q_scale, r_scale)
            G.groot_quantized_product(R8, r_scale, *served["V"], offsets, p["c"], True, inner)
            G.groot_quantized_linear(inner, *served["U"], offsets, None, False, answer, work)
            stream = torch.empty_like(h)
            G.groot_routed_sum(answer, places, weights, h, stream)
            h = stream
        logits = empty(n, CLASSES, like=h)
        G.groot_grouped_product(h, Wo, None, bo, False, logits)
        return logits


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, default=8)
    ap.add_argument("--infer-bits", type=int, default=32)
    ap.add_argument("--epochs", type=int, default=200)
    a = ap.parse_args()
    small, big = Multiplier(a.bits), Multiplier(a.infer_bits, transposed=False)
    model = RoutedClassifier(small.X.shape[1])
    first, last = train(model, small, a.epochs)
    busy = [torch.diff(o).tolist() for o in model.offsets]
    print(f"{a.bits}-bit multiplier, {a.epochs} epochs: loss {first:.4f} -> {last:.4f}; nodes of each expert {busy}")
    with torch.no_grad():
        print(f"{a.infer_bits}-bit multiplier, {big.X.shape[0]} nodes: accuracy {accuracy(model(big), big):.4f} in fp32, "
              f"{accuracy(ServedRouted(model)(big), big):.4f} with experts in 8 bits")


if __name__ == "__main__":
    main()
