"""A node classifier whose weights differ by node type, trained and served through the library.

The nodes of an And-Inverter Graph are primary inputs, AND gates and primary outputs, one kind after the other, so a layer
H = relu((A_hat X) Wn[t] + X Ws[t] + b[t]) with weights for every type t is an aggregation and two grouped products.  Training runs
the aggregation and its transpose, the grouped products and their gradients, and AdamW with states in 8 bits; serving runs the same
layers with the trained weights cut to 8 bits, on a larger multiplier than the model was trained on.

    python examples/typed_classifier.py --bits 8 --infer-bits 64 --epochs 300 --states 8
"""
import argparse
import os
import sys

import numpy as np
import torch
from torch.autograd.function import once_differentiable

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
import paper_2511_18297_amd as G  # noqa: E402
import workloads as wl  # noqa: E402

HIDDEN, CLASSES, THRESHOLD = 32, 5, 32


class Multiplier:
    """Graph, plans, features, labels and the rows of each node type of an n-bit carry-save multiplier."""

    def __init__(self, bits, transposed=True):
        aig = wl.csa_multiplier_aig(bits)
        self.graph = G.groot_graph_build(aig.type, aig.fanin0, aig.fanin1, 1)
        self.plan = G.groot_spmm_plan(self.graph, THRESHOLD)
        G.groot_plan_upload(self.plan, HIDDEN)
        if transposed:
            self.graph_t = G.groot_graph_transpose(self.graph)
            self.plan_t = G.groot_spmm_plan(self.graph_t, THRESHOLD)
            G.groot_plan_upload(self.plan_t, HIDDEN)
        kind = np.asarray(aig.type)
        ends = [0] + [int(i) + 1 for i in np.flatnonzero(np.diff(kind))] + [len(kind)]
        assert len(ends) == 4, "inputs, gates and outputs lie one after the other"
        self.offsets = torch.tensor(ends, dtype=torch.int64, device="cuda")
        self.types = 3
        self.X = torch.from_numpy(wl.paper_node_features(aig)).cuda()
        self.y = torch.from_numpy(aig.label.astype(np.int64)).cuda()


class Aggregate(torch.autograd.Function):
    """Y = A_hat X, dX = A_hat^T dY"""

    @staticmethod
    def forward(ctx, X, m):
        ctx.m, X = m, X.contiguous()
        Y = torch.empty_like(X)
        G.groot_spmm_execute(m.plan, X, Y)
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        dY = dY.contiguous()
        dX = torch.empty_like(dY)
        G.groot_spmm_execute(ctx.m.plan_t, dY, dX)
        return dX, None


class Typed(torch.autograd.Function):
    """Y[i] = X[i] W[t] + b[t] for the rows i of every node type t"""

    @staticmethod
    def forward(ctx, X, W, b, offsets):
        X = X.contiguous()
        Y = torch.empty((X.shape[0], W.shape[2]), dtype=X.dtype, device="cuda")
        G.groot_grouped_product(X, W, offsets, b, False, Y)
        ctx.save_for_backward(X, W, offsets)
        ctx.bias = b is not None
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        X, W, offsets = ctx.saved_tensors
        dY = dY.contiguous()
        dX = dW = db = None
        if ctx.needs_input_grad[0]:
            dX = torch.empty_like(X)
            G.groot_grouped_product_backward_data(dY, W, offsets, dX)
        if ctx.needs_input_grad[1] or ctx.needs_input_grad[2]:
            dW = torch.empty_like(W)
            db = torch.empty((W.shape[0], W.shape[2]), dtype=W.dtype, device="cuda") if ctx.bias else None
            need = G.groot_grouped_product_backward_weights_workspace(X.shape[0], *W.shape, X.dtype)
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
            G.groot_grouped_product_backward_weights(X, dY, offsets, dW, db, workspace)
        return dX, dW, db, None


class TypedClassifier:
    """Two typed layers and a typed output layer."""

    def __init__(self, features, types=3, seed=7):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dims = [(features, HIDDEN), (HIDDEN, HIDDEN), (HIDDEN, CLASSES)]

        def weights(a, b):
            return ((torch.rand((types, a, b), generator=gen, device="cuda") - 0.5) * (2.0 / np.sqrt(a))).requires_grad_(True)
        self.layers = [(weights(a, b), weights(a, b), torch.zeros((types, b), device="cuda", requires_grad=True)) for a, b in dims]

    def parameters(self):
        return [p for layer in self.layers for p in layer]

    def __call__(self, m):
        h = m.X
        for i, (wn, ws, b) in enumerate(self.layers):
            h = Typed.apply(Aggregate.apply(h, m), wn, None, m.offsets) + Typed.apply(h, ws, b, m.offsets)
            h = torch.relu(h) if i + 1 < len(self.layers) else h
        return h


class AdamW:
    """The library's step over all parameters, states in 32 or 8 bits."""

    def __init__(self, params, lr, states=8, weight_decay=1e-4):
        self.params, self.lr, self.weight_decay, self.step_count = params, lr, weight_decay, 0
        zeros = lambda p, dtype: torch.zeros(p.numel(), device="cuda").to(dtype)  # noqa: E731
        self.grads = [torch.zeros_like(p) for p in params]
        kind, more = torch.float32, {}
        if states == 8:
            kind = torch.float8_e4m3fn
            more = {k: [torch.zeros(-(-p.numel() // 256), device="cuda") for p in params] for k in ("m_scale", "v_scale")}
        for p, g in zip(params, self.grads):
            p.grad = g                                       # autograd adds into these
        self.tensors = G.groot_adamw_tensors([p.detach() for p in params], self.grads, [zeros(p, kind) for p in params],
                                             [zeros(p, kind) for p in params], **more)

    def zero_grad(self):
        torch._foreach_zero_(self.grads)

    def step(self):
        self.step_count += 1
        G.groot_adamw_step(self.tensors, self.step_count, self.lr, 0.9, 0.99, 1e-8, self.weight_decay, seed=1)


def train(model, m, epochs, lr=1e-2, states=8):
    """(first loss, last loss) of full-graph training with classes weighted by how rare they are."""
    counts = torch.bincount(m.y, minlength=CLASSES).float()
    weight = counts.sum() / (CLASSES * counts.clamp(min=1))
    opt = AdamW(model.parameters(), lr, states)
    losses = []
    for _ in range(epochs):
        opt.zero_grad()
        loss = torch.nn.functional.cross_entropy(model(m), m.y, weight=weight)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    return float(losses[0]), float(losses[-1])


class Served:
    """The trained layers with their weights in 8 bits, one scale for every type and output channel."""

    def __init__(self, model):
        self.layers = [(self.cut(wn), self.cut(ws), b.detach()) for wn, ws, b in model.layers]

    @staticmethod
    def cut(w):
        types, K, N = w.shape
        rows = w.detach().transpose(1, 2).reshape(types * N, K).contiguous()
        Q, scale = torch.empty((types * N, K), dtype=torch.int8, device="cuda"), torch.empty(types * N, device="cuda")
        G.groot_quantize_rows(rows, Q, scale)
        return Q.view(types, N, K), scale.view(types, N)

    def __call__(self, m):
        h = m.X
        n = h.shape[0]
        workspace = torch.empty(G.groot_quantized_linear_workspace(n, HIDDEN), dtype=torch.uint8, device="cuda")
        for i, (wn, ws, b) in enumerate(self.layers):
            agg = torch.empty_like(h)
            G.groot_spmm_execute(m.plan, h, agg)
            near, own = (torch.empty((n, b.shape[1]), device="cuda") for _ in range(2))
            G.groot_quantized_linear(agg, *wn, m.offsets, None, False, near, workspace)
            G.groot_quantized_linear(h, *ws, m.offsets, b, False, own, workspace)
            h = torch.relu(near + own) if i + 1 < len(self.layers) else near + own
        return h


def accuracy(logits, m):
    return float((logits.argmax(1) == m.y).float().mean())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--bits", type=int, default=8)
    ap.add_argument("--infer-bits", type=int, default=64)
    ap.add_argument("--epochs", type=int, default=300)
    ap.add_argument("--states", type=int, choices=(8, 32), default=8)
    a = ap.parse_args()
    small, big = Multiplier(a.bits), Multiplier(a.infer_bits, transposed=False)
    model = TypedClassifier(small.X.shape[1])
    first, last = train(model, small, a.epochs, states=a.states)
    print(f"{a.bits}-bit multiplier, {a.epochs} epochs, AdamW states in {a.states} bits: loss {first:.4f} -> {last:.4f}")
    with torch.no_grad():
        print(f"{a.infer_bits}-bit multiplier, {big.X.shape[0]} nodes: accuracy {accuracy(model(big), big):.4f} in fp32, "
              f"{accuracy(Served(model)(big), big):.4f} with layers in 8 bits")


if __name__ == "__main__":
    main()
