"""The routed layer as the README prints it: its lines are run, and what they leave is compared with autograd in 64 bits."""
import os
import re

import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def printed(heading, behind):
    """the indented lines between the paragraphs that begin with `heading` and with `behind`"""
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    part = text[text.index(heading):text.index(behind)]
    return "\n".join(line[4:] for line in part.splitlines() if re.match(r"    \S", line))


def test_the_routed_layer():
    """Sums of up to 300 products in fp32 lose 300 x 2^-24 of their terms' magnitudes at the most, and a path has ten of them: 2^-12 of these.  2^-10 of the
    largest value leaves four times that for terms that cancel."""
    n, K, inner, E, k = 300, 32, 48, 16, 3
    gen = torch.Generator(device="cuda").manual_seed(400)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * scale
    given = dict(x=normal(n, K), stream=normal(n, K), gain=1 + normal(K, scale=0.2), Wr=normal(1, K, E, scale=0.3), V=normal(E, K, inner, scale=0.2), c=normal(E, inner),
                 U=normal(E, inner, K, scale=0.2), dout=normal(n, K))
    before = {name: t.clone() for name, t in given.items()}

    def empty(*shape):
        return torch.full(shape, float("nan"), device="cuda")
    buffers = dict(y=empty(n, K), rstd=empty(n), scores=empty(n, E), weights=empty(n, k), R=empty(n * k, K), Z=empty(n * k, inner), A=empty(n * k, K), out=empty(n, K),
                   dA=empty(n * k, K), dZ=empty(n * k, inner), dR=empty(n * k, K), dweights=empty(n, k), dscores=empty(n, E), dy=empty(n, K), dy_scores=empty(n, K),
                   dx=empty(n, K), dgain=empty(K), dWr=empty(1, K, E), dV=empty(E, K, inner), dc=empty(E, inner), dU=empty(E, inner, K), bias=normal(E, scale=0.05),
                   chosen=torch.zeros((n, k), dtype=torch.int32, device="cuda"), places=torch.zeros((n, k), dtype=torch.int32, device="cuda"),
                   offsets=torch.zeros(E + 1, dtype=torch.int64, device="cuda"))
    work = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    names = dict(given, **buffers, G=G, workspace=work, route_work=work, weight_work=work, norm_work=work)
    exec(printed("A routed layer (", "Layout:"), names)

    p = {name: before[name].cpu().double().requires_grad_(name != "dout") for name in before}
    h = p["x"] + p["stream"]
    y = h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6) * p["gain"]
    chosen = names["chosen"].cpu().long()
    w = torch.gather(torch.sigmoid(y @ p["Wr"][0]), 1, chosen)
    w = w / w.sum(1, keepdim=True)
    z = torch.relu(torch.einsum("nk,nskj->nsj", y, p["V"][chosen]) + p["c"][chosen])
    out = h + (torch.einsum("nsj,nsjk->nsk", z, p["U"][chosen]) * w[:, :, None]).sum(1)
    want = dict(zip(("x", "gain", "Wr", "V", "c", "U"), torch.autograd.grad(out, [p[name] for name in ("x", "gain", "Wr", "V", "c", "U")], p["dout"])))
    for name, got, exact in [("out", names["out"], out.detach())] + [("d" + name, names["d" + name], g) for name, g in want.items()]:
        err = (got.cpu().double() - exact).abs().max()
        assert float(err) <= 2.0 ** -10 * float(exact.abs().max()), name
