"""The weights of a choice and their gradient, to the last place whatever the spread of the scores.

Weights are computed in 64 bits and rounded once: half a step of fp32, u = 2^-24 of the value (2^-150 below 2^-126), and 2^-29 of the value for what
64 bits and the exponential's series leave.  But for one sum: that of a softmax over all experts, where neither a bias decides nor weights are
renormalised, has terms p in fp32.  x below the largest score, x is rounded once, its product with a rounded log2(e) twice and the exponential to a step: p is
off by (2.5 |x| + 2) u, and in pairs over 16 values and up to 64 lanes every term meets 10 additions: (2.5 sum p |x| + 12) u.
Gradients: every term is computed in 64 bits and rounded to fp32 where it waits, so with the difference's own rounding, and the row's common
factor's, four roundings of the terms' magnitudes, 4 u, and one rounding to the type; with that sum, its error and (2.5 |x| + 2) u of every p more.
"""
import math

import numpy as np
import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402
from test_gpu_routed import GATES, LEAST, TYPES, UNIT, check_route, how, own_route  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# experts, top k: every length of the lists, and more slots than they hold
SIZES = [(8, 3), (16, 16), (33, 5), (128, 8), (256, 12), (400, 20), (1024, 32)]


def scores_of(E, dtype, spread, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((200, E), generator=gen, device="cuda") * spread).to(dtype), torch.randn(E, generator=gen, device="cuda") * 0.05


def chosen_log(x, gate):
    return x if gate == "softmax" else np.minimum(x, 0) - np.log1p(np.exp(-np.abs(x)))


def sum_error(x):
    """of a softmax's sum in fp32, for every row, relative"""
    m = x.max(1, keepdims=True)
    p = np.exp(x - m) / np.exp(x - m).sum(1, keepdims=True)
    return (2.5 * (p * (m - x)).sum(1, keepdims=True) + 12) * U


def exact_weights(scores, experts, gate, renormalise, factor):
    x, e = scores.double().cpu().numpy(), experts.long().cpu().numpy()
    u = np.take_along_axis(chosen_log(x, gate), e, 1)
    if renormalise:
        q = np.exp(u - u.max(1, keepdims=True))
        return factor * q / q.sum(1, keepdims=True)
    if gate == "sigmoid":
        return factor * np.exp(u)
    m = x.max(1, keepdims=True)
    return factor * np.exp(u - m) / np.exp(x - m).sum(1, keepdims=True)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
@pytest.mark.parametrize("biased", (False, True))
@pytest.mark.parametrize("spread", (1.0, 20.0, 300.0))
def test_weights_are_rounded_once(kind, gate, renormalise, biased, spread):
    for E, k in SIZES:
        scores, bias = scores_of(E, TYPES[kind], spread, 600 + E)
        for factor in (1.0, 0.1):
            experts, weights, _, _ = own_route(scores, bias if biased else None, k, **how(gate, renormalise=renormalise, factor=factor))
            assert bool((experts >= 0).all())
            want = torch.from_numpy(exact_weights(scores, experts, gate, renormalise, factor)).cuda()
            whole = gate == "softmax" and not renormalise and not biased
            more = torch.from_numpy(sum_error(scores.double().cpu().numpy())).cuda() if whole else 0.0
            err, bound = (weights.double() - want).abs(), (U + 2.0 ** -29 + more) * want + 2.0 ** -150
            assert bool((err <= bound).all()), f"{E} experts, top {k}, factor {factor}: {float((err / want.clamp(min=1e-300) / U)[err > bound].max())} half steps"


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
@pytest.mark.parametrize("spread", (1.0, 20.0, 300.0))
def test_gradients_of_scores_far_apart(kind, gate, renormalise, spread):
    T, factor = TYPES[kind], 0.1
    for E, k in SIZES:
        scores, _ = scores_of(E, T, spread, 650 + E)
        experts = own_route(scores, None, k, **how(gate, renormalise=renormalise))[0]
        dw = torch.randn((200, k), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
        ds = torch.full_like(scores, math.nan)
        G.groot_route_backward(scores, experts, dw, ds, gate=GATES[gate], renormalise=renormalise, factor=factor)
        x, e, d = scores.double().cpu().numpy(), experts.long().cpu().numpy(), dw.double().cpu().numpy()
        w = exact_weights(scores, experts, gate, renormalise, factor)
        part, whole = np.zeros_like(x), np.zeros_like(x)      # of the logarithms of the chosen probabilities
        np.put_along_axis(part, e, w * (d - (w * d).sum(1, keepdims=True) / factor) if renormalise else w * d, 1)
        np.put_along_axis(whole, e, w * (np.abs(d) + (w * np.abs(d)).sum(1, keepdims=True) / factor) if renormalise else w * np.abs(d), 1)
        if gate == "sigmoid":
            left = np.exp(chosen_log(-x, gate))                # 1 - p
            part, whole = part * left, whole * left
        elif not renormalise:
            m = x.max(1, keepdims=True)
            p = np.exp(x - m) / np.exp(x - m).sum(1, keepdims=True)
            off, mean = sum_error(x) / U, p * whole.sum(1, keepdims=True)
            part, whole = part - p * part.sum(1, keepdims=True), whole * (1 + off / 4) + mean * (1 + off / 2 + (2.5 * (m - x) + 2) / 4)
        want, terms = torch.from_numpy(part).cuda(), torch.from_numpy(whole).cuda()
        err, bound = (ds.double() - want).abs(), 4 * U * terms + 1.01 * UNIT[T] * want.abs() + 2 * LEAST[T]
        assert bool((err <= bound).all()), f"{E} experts, top {k}: {float((err / bound).max())} of the tolerance"


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
@pytest.mark.parametrize("sets", ((1, 1, 1), (4, 3, 2)))
@pytest.mark.parametrize("E, k", [(24, 18), (48, 24), (400, 17), (1024, 32)])
def test_many_slots_of_masked_rows(gate, renormalise, sets, E, k):
    """more slots than a row has experts left, rows without one, infinities and NaN"""
    scores, bias = scores_of(E, torch.float32, 2.0, 700 + E)
    scores[3] = -math.inf
    scores[4, 1:] = -math.inf
    scores[5, k - 2:] = -math.inf
    scores[6, : E - 3] = -math.inf
    scores[7, 3], scores[8, 5], scores[9] = math.nan, math.inf, math.nan
    scores[10] = torch.finfo(torch.float32).min
    scores[11, 1:] = torch.finfo(torch.float32).min
    scores[150:] = -math.inf
    check_route(scores, None, k, **how(gate, *sets, renormalise))
    bias[0], bias[1], bias[2] = -math.inf, math.nan, 3.0
    if gate == "sigmoid":
        scores[10] = 2.0                                     # values of 0 and of numbers next to it are no values of their own with a bias
        scores[11, 1:] = 1.0
    check_route(scores, bias, k, **how(gate, *sets, renormalise))
