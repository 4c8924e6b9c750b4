"""Routing to experts and the rows' way there and back, against plain implementations in 64 bits.

Experts, places and offsets have to be equal.  Tolerances of the rest, from the arithmetic that the calls state (u = 2^-24, half a step of
fp32):
  * a weight is exp(x - m) over a sum of at most E such terms.  x - m is rounded once, which changes exp by at most |x - m| u relative, and
    exp, the logarithm of the sigmoid, the quotient and the factor are within 4 u each; every addition of the sum loses at most u, and at most 16
    + log2(64) of them lie on one term's way, as lanes add up to 16 terms each and meet pairwise: (|x - m| + 40) 2 u, and 2^-126 where it
    underflows.  dscores are sums of two products of such weights and given gradients: twice that of their terms' magnitudes, and one rounding.
  * sum: k products and additions in fp32: (k + 2) 2 u of the terms' magnitudes, one rounding to the type (fp32 2^-24, bf16 2^-8, fp16 2^-11 of the
    value).  dweights: K terms: (K + 2) 2 u of their magnitudes at the most.
"""
import math

import numpy as np
import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
U2 = 2.0 ** -23
NAN, INF = float("nan"), float("inf")
BIAS = 11399345 * 2.0 ** -54                               # 0.68 x 2^-30, held by fp32
GATES = {"softmax": G.GROOT_SOFTMAX, "sigmoid": G.GROOT_SIGMOID}


# ---------------------------------------------------------------------------------------------------------------
# the choice, row by row, in Python's 64-bit numbers
# ---------------------------------------------------------------------------------------------------------------
def probabilities(x, gate):
    if gate == "sigmoid":
        return np.array([1 / (1 + math.exp(-v)) if v > -700 else 0.0 for v in x])
    m = x.max()
    e = np.exp(x - (m if np.isfinite(m) else 0.0))
    with np.errstate(invalid="ignore"):
        return e / e.sum()


def route_row(x, bias, k, gate, sets, open_sets, set_best, renormalise, factor):
    """(experts, weights, magnitude of the largest x - m on the way) of one row of scores"""
    E = len(x)
    if np.isnan(x).any() or (gate == "softmax" and (x == INF).any()):
        return [-1] * k, [NAN] * k
    p = probabilities(x, gate)
    c = x.copy() if bias is None and set_best == 1 else p + (bias if bias is not None else 0.0)
    c[(x == -INF) | ~(c > -INF)] = -INF
    if open_sets < sets:
        size = E // sets
        value = []
        for s in range(sets):
            best = sorted(c[s * size:(s + 1) * size], reverse=True)[:set_best]
            value.append(-INF if best[0] == -INF else sum(v for v in best if v > -INF))
        order = sorted(range(sets), key=lambda s: (-value[s], s))
        for s in order[open_sets:]:
            c[s * size:(s + 1) * size] = -INF
    order = [e for e in sorted(range(E), key=lambda e: (-c[e], e)) if c[e] > -INF][:k]
    if renormalise:
        u = [x[e] if gate == "softmax" else min(x[e], 0.0) - math.log1p(math.exp(-abs(x[e]))) for e in order]
        q = [math.exp(v - max(u)) for v in u]
        w = [factor * v / sum(q) for v in q]
    else:
        w = [factor * p[e] for e in order]
    pad = k - len(order)
    return order + [-1] * pad, w + [0.0] * pad


def route_plain(scores, bias, k, **how):
    x = scores.double().cpu().numpy()
    b = None if bias is None else bias.double().cpu().numpy()
    rows = [route_row(r, b, k, **how) for r in x]
    experts = np.array([r[0] for r in rows], dtype=np.int64).reshape(-1, k)
    weights = np.array([r[1] for r in rows], dtype=np.float64).reshape(-1, k)
    E = scores.shape[1]
    offsets = np.concatenate([[0], np.cumsum(np.bincount(experts[experts >= 0], minlength=E))])
    places = np.full(experts.shape, -1, dtype=np.int64)
    nxt = offsets[:-1].copy()
    for i, row in enumerate(experts):
        for s, e in enumerate(row):
            if e >= 0:
                places[i, s] = nxt[e]
                nxt[e] += 1
    return experts, weights, places, offsets


def buffers(n, E, k):
    full = lambda *shape, value, type: torch.full(shape, value, dtype=type, device="cuda")  # noqa: E731
    return (full(n, k, value=-7, type=torch.int32), full(n, k, value=NAN, type=torch.float32), full(n, k, value=-7, type=torch.int32),
            full(E + 1, value=-7, type=torch.int64))


def workspace(bytes):
    return torch.full((max(bytes, 16),), 0x5A, dtype=torch.uint8, device="cuda")


def own_route(scores, bias, k, gate, sets, open_sets, set_best, renormalise, factor, **more):
    n, E = scores.shape
    out = buffers(n, E, k)
    G.groot_route(scores, bias, *out, workspace(G.groot_route_workspace(n, E, k)), gate=GATES[gate], sets=sets, open_sets=open_sets, set_best=set_best,
                  renormalise=renormalise, factor=factor, **more)
    return out


def reach(scores):
    """the largest |x - m| of a row's finite scores, for the weights' tolerance"""
    x = scores.double()
    fine = torch.isfinite(x)
    most = torch.where(fine, x, torch.full_like(x, -INF)).amax(1, keepdim=True)
    far = torch.where(fine, (x - most).abs().clamp(max=200.0), torch.zeros_like(x)).amax(1, keepdim=True)
    return torch.maximum(far, torch.where(fine, x.abs().clamp(max=200.0), torch.zeros_like(x)).amax(1, keepdim=True))


def check_route(scores, bias, k, **how):
    got = own_route(scores, bias, k, **how)
    want = route_plain(scores, bias, k, **how)
    for name, g, w in (("experts", got[0], want[0]), ("places", got[2], want[2]), ("offsets", got[3], want[3])):
        g = g.cpu().numpy()
        assert np.array_equal(g, w), f"{name}: first at {np.argwhere(g != w)[0]}, {g[tuple(np.argwhere(g != w)[0])]} for {w[tuple(np.argwhere(g != w)[0])]}"
    g, w = got[1].double().cpu(), torch.from_numpy(want[1])
    assert torch.equal(torch.isnan(g), torch.isnan(w)), "weights: NaN"
    bound = (reach(scores).cpu() + 40) * U2 * w.abs() + abs(how["factor"]) * LEAST[torch.float32]
    bad = ~torch.isnan(w) & ~((g - w).abs() <= bound)
    assert not bad.any(), f"weights: {int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}: {g[bad][0]} for {w[bad][0]}"
    return got


def made(n, E, dtype, seed, spread=1.5, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn((max(n, 1), E + pad), generator=gen, device="cuda") * spread + torch.randn(E + pad, generator=gen, device="cuda") * 0.5
    bias = torch.randn(E, generator=gen, device="cuda") * 0.1
    return wide.to(dtype)[:n, pad // 2:pad // 2 + E], bias


def how(gate="softmax", sets=1, open_sets=1, set_best=1, renormalise=True, factor=1.0):
    return dict(gate=gate, sets=sets, open_sets=open_sets, set_best=set_best, renormalise=renormalise, factor=factor)


# rows, experts, k, bias, more columns, the rest
CASES = [
    (1, 1, 1, False, 0, how()),
    (1, 64, 4, False, 0, how()),
    (3, 2, 2, True, 1, how("sigmoid", renormalise=False, factor=2.5)),
    (64, 8, 2, False, 0, how()),
    (65, 8, 2, True, 0, how("sigmoid")),
    (128, 256, 8, True, 0, how("sigmoid", 8, 4, 2, True, 2.5)),
    (63, 160, 6, False, 3, how("softmax", 8, 3, 1, False, 16.0)),
    (200, 17, 17, True, 5, how("softmax")),
    (130, 15, 15, False, 0, how("sigmoid", 5, 5, 2)),
    (70, 30, 3, True, 0, how("softmax", 10, 1, 2, False)),
    (300, 257, 5, False, 7, how("sigmoid", factor=0.5)),
    (129, 512, 12, True, 0, how("softmax", 64, 7, 2)),
    (67, 1024, 32, True, 0, how("sigmoid", 16, 3, 2)),
    (40, 1000, 1, False, 0, how("softmax", 4, 1, 1, False)),
    (90, 100, 20, True, 0, how("sigmoid", 20, 9, 1)),
    (1000, 128, 8, False, 0, how()),
    (4200, 16, 1, True, 0, how("softmax", 2, 1, 2, False)),
    (70, 64, 32, False, 0, how("softmax", 64, 40, 1)),
    (5000, 33, 3, False, 0, how("sigmoid", 3, 2, 2)),
]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_route(kind, case):
    n, E, k, biased, pad, rest = CASES[case]
    scores, bias = made(n, E, TYPES[kind], 300 + case, pad=pad)
    check_route(scores, bias if biased else None, k, **rest)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("biased", (False, True))
@pytest.mark.parametrize("sets", ((1, 1, 1), (4, 2, 1), (4, 2, 2)))
def test_ties_go_to_the_lowest(gate, biased, sets):
    """scores and bias of a few values: many experts, and sets, of the same value"""
    gen = torch.Generator(device="cuda").manual_seed(11)
    for E, k in ((32, 6), (64, 16), (512, 9)):
        scores = torch.randint(0, 3, (150, E), generator=gen, device="cuda").float()
        scores[0] = 0
        # two sums of the same four numbers round differently: where sums are compared, all have one bias
        bias = torch.full((E,), 0.25, device="cuda") if sets[2] == 2 else torch.randint(0, 2, (E,), generator=gen, device="cuda").float() * 0.25
        check_route(scores, bias if biased else None, k, **how(gate, *sets))


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
@pytest.mark.parametrize("biased", (False, True))
def test_values_next_to_each_other(gate, renormalise, biased):
    """fp32 scores a step or a few apart, where only 64 bits tell the values of the choice apart; the bias is no multiple of a step of the
    probabilities near 1 / 48 (2^-30 is three of them, and sums that are equal in exact numbers round apart)"""
    gen = torch.Generator(device="cuda").manual_seed(12)
    base = torch.randn((120, 1), generator=gen, device="cuda")
    steps = torch.randint(-3, 4, (120, 48), generator=gen, device="cuda").float()
    scores = base * (1 + steps * 2.0 ** -23)
    bias = torch.randint(0, 2, (48,), generator=gen, device="cuda").float() * BIAS if biased else None
    # numbers in 64 bits lie 2^-53 apart: values that come closer than a few of these could fall either way, equal ones cannot
    x = scores.double().cpu().numpy()
    for row in x:
        c = np.sort(np.unique(probabilities(row, gate)[:, None] + (np.array([0.0, BIAS]) if biased else np.array([0.0]))))
        assert np.diff(c).size == 0 or np.diff(c).min() > 2.0 ** -48
    check_route(scores, bias, 7, **how(gate, renormalise=renormalise))
    check_route(scores, bias, 7, **how(gate, 6, 3, 1, renormalise))


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
@pytest.mark.parametrize("sets", ((1, 1, 1), (4, 2, 1), (4, 2, 2)))
@pytest.mark.parametrize("E", (24, 400))
def test_masks_infinities_and_nan(gate, renormalise, sets, E):
    scores, bias = made(140, E, torch.float32, 21)
    scores = scores.contiguous()
    scores[3] = -INF                                       # nothing is left
    scores[4, 1:] = -INF                                   # one expert
    scores[5, 2:] = -INF                                   # fewer than k
    scores[6, :E // 2] = -INF                              # half of the sets
    scores[7, E // 4 + 1:] = -INF                          # a set and one expert more
    scores[8, 3] = NAN
    scores[9, 5] = INF
    scores[10] = NAN
    scores[11] = -INF
    scores[11, 2] = NAN
    scores[12] = torch.finfo(torch.float32).min            # a mask of the type's lowest value is no mask
    scores[13, 1:] = torch.finfo(torch.float32).min
    scores[14] = -200.0                                    # probabilities that fp32 does not hold
    scores[15] = 90.0
    scores[100:] = -INF                                    # a padded batch
    check_route(scores, None, 5, **how(gate, *sets, renormalise))
    if gate == "sigmoid":
        scores[14], scores[15] = 0.0, 1.0                  # with a bias, values of 1e-87 and of 1 - 1e-39 are no values of their own in 64 bits
        scores[12] = 2.0
    bias[0], bias[1], bias[2] = -INF, NAN, 3.0
    check_route(scores, bias, 5, **how(gate, *sets, renormalise))
    bias[:] = -INF
    got = check_route(scores, bias, 5, **how(gate, *sets, renormalise))
    assert int(got[3][-1]) == 0


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("sets", ((1, 1, 1), (6, 2, 1), (6, 2, 2), (24, 4, 2), (3, 1, 2), (8, 3, 2), (2, 1, 2)))
def test_a_bias_of_plus_infinity_comes_first(gate, sets):
    """experts with it tie with one another, as their sets do, and are closed where their score is -inf"""
    scores, bias = made(140, 48, torch.float32, 22)
    bias[7], bias[30], bias[31] = INF, INF, INF
    scores[::3, 30] = -INF
    check_route(scores, bias, 2, **how(gate, *sets, True))
    bias[:] = INF
    bias[40] = torch.finfo(torch.float32).min
    check_route(scores, bias, 2, **how(gate, *sets, False))


def test_no_rows():
    for E in (8, 600):
        got = own_route(torch.empty((0, E), device="cuda"), None, 2, **how())
        assert torch.equal(got[3], torch.zeros(E + 1, dtype=torch.int64, device="cuda"))


def test_many_rows_are_in_order():
    """more workgroups than one scan's threads; checked by what the places mean"""
    scores, bias = made(70001, 64, torch.bfloat16, 31)
    scores[69000:] = -INF
    experts, weights, places, offsets = own_route(scores, bias, 6, **how("sigmoid", 8, 4, 2))
    flat = experts.reshape(-1).long()
    order = torch.sort(torch.where(flat < 0, torch.full_like(flat, 99), flat), stable=True).indices[:69000 * 6]
    assert torch.equal(places.reshape(-1)[order].long(), torch.arange(69000 * 6, device="cuda"))
    assert int((places[69000:] != -1).sum()) == 0 and int((experts[69000:] != -1).sum()) == 0
    assert torch.equal(offsets[1:], torch.cumsum(torch.bincount(flat[flat >= 0], minlength=64), 0)) and int(offsets[0]) == 0
    assert torch.equal((weights == 0).all(1), torch.arange(70001, device="cuda") >= 69000)
    # the same rows alone have the same experts and weights
    few = own_route(scores[500:520], bias, 6, **how("sigmoid", 8, 4, 2))
    assert torch.equal(few[0], experts[500:520]) and torch.equal(few[1], weights[500:520])


# ---------------------------------------------------------------------------------------------------------------
# the gradient of the scores
# ---------------------------------------------------------------------------------------------------------------
def weights64(x, experts, gate, renormalise, factor):
    """the chosen weights as a function of the scores, in 64 bits, differentiable"""
    taken = experts >= 0
    at = experts.clamp(min=0)
    if renormalise:
        u = torch.gather(x if gate == "softmax" else torch.nn.functional.logsigmoid(x), 1, at)
        w = factor * torch.softmax(torch.where(taken, u, torch.full_like(u, -1e300)), 1)
    else:
        w = factor * torch.gather(torch.softmax(x, 1) if gate == "softmax" else torch.sigmoid(x), 1, at)
    return torch.where(taken, w, torch.zeros_like(w))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
@pytest.mark.parametrize("n, E, k, pad", [(1, 1, 1, 0), (1, 64, 4, 0), (77, 5, 2, 1), (130, 40, 16, 3), (65, 256, 8, 0), (90, 300, 3, 0), (33, 1024, 32, 5), (3000, 64, 6, 0)])
def test_route_backward(kind, gate, renormalise, n, E, k, pad):
    dtype, factor = TYPES[kind], 2.5
    scores, _ = made(n, E, dtype, 41, pad=pad)
    if E > 8 and n > 8:
        scores[5], scores[6, 2:], scores[7, ::3] = -INF, -INF, -INF
    experts = own_route(scores, None, k, **how(gate, renormalise=renormalise))[0]
    dw = torch.randn((n, k), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    ds = torch.full((n, E + pad), NAN, device="cuda").to(dtype)[:, :E]
    G.groot_route_backward(scores, experts, dw, ds, gate=GATES[gate], renormalise=renormalise, factor=factor)
    # -inf takes no part: a score so low that its exponential is 0 has the same weights, and no gradient
    x = torch.where(torch.isinf(scores), torch.full_like(scores, 0).double() - 1e6, scores.double()).cpu().requires_grad_(True)
    e = experts.long().cpu()
    w = weights64(x, e, gate, renormalise, factor)
    w.backward(dw.double().cpu())
    want = torch.where(torch.isinf(scores.cpu()), torch.zeros_like(x), x.grad)
    # the terms: own weight x own gradient, and the row's mean for everybody whom the sum holds
    own = torch.zeros_like(x).scatter_add_(1, e.clamp(min=0), (w * dw.double().cpu()).abs().detach())
    mean = (w * dw.double().cpu()).abs().sum(1, keepdim=True).detach()
    share = torch.softmax(x.detach(), 1) if gate == "softmax" and not renormalise else torch.zeros_like(x).scatter_add_(1, e.clamp(min=0), w.detach() / factor)
    terms = own + share * mean
    bound = 2 * (reach(scores).cpu() + 40) * U2 * terms + UNIT[dtype] * want.abs() * 1.01 + LEAST[dtype] * 8
    bad = ~((ds.double().cpu() - want).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}: {ds.double().cpu()[bad][0]} for {want[bad][0]}"


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
def test_route_backward_by_differences(gate, renormalise):
    """sum w dw moves by h times the gradient along a direction, to h^2 (difference of both sides, in 64 bits)"""
    scores, _ = made(50, 24, torch.float32, 51)
    experts = own_route(scores, None, 5, **how(gate, renormalise=renormalise))[0]
    gen = torch.Generator(device="cuda").manual_seed(6)
    dw, along = torch.randn((50, 5), generator=gen, device="cuda"), torch.randn((50, 24), generator=gen, device="cuda").double()
    ds = torch.empty_like(scores)
    G.groot_route_backward(scores, experts, dw, ds, gate=GATES[gate], renormalise=renormalise)
    h, e = 1e-4, experts.long()
    value = [(weights64(scores.double() + s * h * along, e, gate, renormalise, 1.0) * dw.double()).sum(1) for s in (1, -1)]
    got, want = (ds.double() * along).sum(1), (value[0] - value[1]) / (2 * h)
    # the third derivative of a weight is below 1 in each direction's scores: |along|_1^3 h^2 / 6, and fp32's rounding of 24 terms
    size = along.abs().sum(1)
    assert bool(((got - want).abs() <= size ** 3 * h * h * dw.abs().sum(1) + 100 * U2 * size * dw.abs().sum(1)).all())


def test_route_backward_of_broken_rows_and_foreign_experts():
    scores, _ = made(6, 20, torch.float32, 61)
    scores[0, 3], scores[1, 2], scores[2] = NAN, INF, -INF
    experts = torch.tensor([[-1, -1], [-1, -1], [-1, -1], [4, 4], [25, 3], [-9, 2]], dtype=torch.int32, device="cuda")
    dw, ds = torch.full((6, 2), 2.0, device="cuda"), torch.empty_like(scores)
    G.groot_route_backward(scores, experts, dw, ds, renormalise=False)
    assert torch.isnan(ds[:2]).all() and bool((ds[2] == 0).all())
    p = torch.softmax(scores[3:].double(), 1)
    for row, chosen in ((0, (4, 4)), (1, (3,)), (2, (2,))):       # an expert named twice counts twice, one that there is not none
        g = torch.zeros(20, dtype=torch.float64, device="cuda")
        for e in chosen:
            g[e] += 2
        want = p[row] * (g - (g * p[row]).sum())
        assert torch.allclose(ds[3 + row].double(), want, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("renormalise", (False, True))
def test_route_backward_of_slots_without_an_expert(gate, renormalise):
    """what stands in their gradient counts for nothing, NaN neither"""
    scores, _ = made(70, 24, torch.bfloat16, 62)
    experts = own_route(scores, None, 5, **how(gate, renormalise=renormalise))[0]
    gen = torch.Generator(device="cuda").manual_seed(7)
    experts = torch.where(torch.rand((70, 5), generator=gen, device="cuda") < 0.4, torch.full_like(experts, -1), experts)
    dw = torch.randn((70, 5), generator=gen, device="cuda")
    results = []
    for there in (0.0, NAN, INF):
        ds = torch.full_like(scores, NAN)
        G.groot_route_backward(scores, experts, torch.where(experts < 0, torch.full_like(dw, there), dw), ds, gate=GATES[gate], renormalise=renormalise)
        results.append(ds)
    assert not torch.isnan(results[0]).any() and all(torch.equal(results[0], r) for r in results[1:])


# ---------------------------------------------------------------------------------------------------------------
# rows and their places
# ---------------------------------------------------------------------------------------------------------------
def dealt(n, k, E, seed, empty=0.2, spare=3):
    """places of n rows in the order of random experts, some slots without one, and the number of rows of R (a few behind the last place)"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    experts = torch.topk(torch.rand((n, E), generator=gen, device="cuda"), k).indices if n else torch.zeros((0, k), dtype=torch.long, device="cuda")
    experts = torch.where(torch.rand((n, k), generator=gen, device="cuda") < empty, torch.full_like(experts, -1), experts).reshape(-1)
    order = torch.sort(torch.where(experts < 0, torch.full_like(experts, E), experts), stable=True).indices
    places = torch.empty_like(experts)
    places[order] = torch.arange(n * k, device="cuda")
    places = torch.where(experts < 0, torch.full_like(experts, -1), places)
    return places.reshape(n, k).int(), int((experts >= 0).sum()) + spare, gen


def matrix(gen, rows, cols, dtype, pad=0, scale=1.0):
    wide = torch.randn((max(rows, 1), cols + pad), generator=gen, device="cuda") * scale
    if dtype == torch.int8:
        wide = torch.clamp(torch.round(wide * 40), -127, 127)
    return wide.to(dtype)[:rows, pad // 2:pad // 2 + cols]


def guarded(rows, cols, dtype, pad=0, value=77.0):
    wide = torch.full((max(rows, 1), cols + pad), value, device="cuda").to(dtype)
    return wide[:rows, pad // 2:pad // 2 + cols], wide


def untouched(wide, view, pad, value=77.0):
    """the columns beside the matrix, as they were"""
    cols = view.shape[1]
    return bool((wide[:, :pad // 2] == torch.tensor(value).to(wide.dtype)).all() and (wide[:, pad // 2 + cols:] == torch.tensor(value).to(wide.dtype)).all())


# rows, k, experts, width, pad
WAYS = [(1, 1, 1, 1, 0), (1, 4, 8, 64, 0), (3, 2, 4, 3, 1), (5, 3, 7, 8, 0), (17, 2, 5, 15, 3), (40, 4, 6, 17, 1), (70, 3, 9, 64, 8), (129, 2, 16, 100, 5), (33, 8, 32, 256, 0),
        (65, 1, 2, 1000, 0), (31, 5, 11, 1001, 7), (20, 32, 40, 513, 0), (300, 2, 8, 2048, 0), (9, 3, 4, 8200, 16), (2, 2, 3, 65536, 0), (2, 6, 6, 20001, 1), (4001, 2, 8, 32, 0)]


@pytest.mark.parametrize("kind", list(TYPES) + ["i8"])
@pytest.mark.parametrize("case", range(len(WAYS)))
def test_rows_to_their_places(kind, case):
    n, k, E, K, pad = WAYS[case]
    dtype = TYPES.get(kind, torch.int8)
    places, m, gen = dealt(n, k, E, 70 + case)
    X = matrix(gen, n, K, dtype, pad)
    scale = torch.rand(n, generator=gen, device="cuda") if case % 2 else None
    R, wide = guarded(m, K, dtype, pad)
    r_scale = torch.full((m,), 77.0, device="cuda") if case % 2 else None
    G.groot_routed_rows(X, places, R, scale, r_scale)
    want = torch.full((m, K), 77.0, device="cuda").to(dtype)
    i, s = torch.nonzero(places >= 0, as_tuple=True)
    at = places[i, s].long()
    want[at] = X[i]
    assert torch.equal(R, want) and untouched(wide, R, pad)
    if case % 2:
        want = torch.full((m,), 77.0, device="cuda")
        want[at] = scale[i]
        assert torch.equal(r_scale, want)


def slots64(R, places):
    rows = R.double()[places.clamp(min=0).long()]
    return torch.where((places >= 0)[:, :, None], rows, torch.zeros((), dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(WAYS)))
@pytest.mark.parametrize("weighted, added", ((True, True), (False, False)))
def test_sum_over_the_places(kind, case, weighted, added):
    n, k, E, K, pad = WAYS[case]
    dtype = TYPES[kind]
    places, m, gen = dealt(n, k, E, 90 + case)
    R = matrix(gen, m, K, dtype, pad)
    R[m - 3:] = NAN                                          # behind the last place
    w = torch.randn((n, k), generator=gen, device="cuda") if weighted else None
    addend = matrix(gen, n, K, dtype, 2 * pad) if added else None
    out, wide = guarded(n, K, dtype, pad)
    G.groot_routed_sum(R, places, w, addend, out)
    parts = slots64(R, places) * (w.double()[:, :, None] if weighted else 1.0)
    first = addend.double() if added else torch.zeros((n, K), dtype=torch.float64, device="cuda")
    want, terms = first + parts.sum(1), first.abs() + parts.abs().sum(1)
    bound = (k + 2) * U2 * terms + UNIT[dtype] * want.abs() * 1.01 + LEAST[dtype]
    err = (out.double() - want).abs()
    assert bool((err <= bound).all()), (err / bound).max()
    assert untouched(wide, out, pad)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(WAYS)))
def test_sum_backward(kind, case):
    n, k, E, K, pad = WAYS[case]
    dtype = TYPES[kind]
    places, m, gen = dealt(n, k, E, 110 + case)
    R, dout = matrix(gen, m, K, dtype, pad), matrix(gen, n, K, dtype, 2 * pad)
    w = torch.randn((n, k), generator=gen, device="cuda")
    for weights, want_rows, want_weights in ((w, True, True), (None, True, True), (w, True, False), (w, False, True)):
        dR, wide = guarded(m, K, dtype, pad)
        dw = torch.full((n, k), NAN, device="cuda")
        G.groot_routed_sum_backward(dout, R if want_weights else None, places, weights, dR if want_rows else None, dw if want_weights else None)
        held = places >= 0
        if want_rows:
            want = torch.full((m, K), 77.0, dtype=torch.float64, device="cuda")
            i, s = torch.nonzero(held, as_tuple=True)
            at = places[i, s].long()
            want[at] = dout.double()[i] * (w.double()[i, s][:, None] if weights is not None else 1.0)
            bound = torch.zeros_like(want)
            bound[at] = 2 * U2 * want[at].abs() + UNIT[dtype] * want[at].abs() * 1.01 + LEAST[dtype]
            assert bool(((dR.double() - want).abs() <= bound).all()) and untouched(wide, dR, pad)
        if want_weights:
            parts = slots64(R, places) * dout.double()[:, None, :]
            bound = (K + 2) * U2 * parts.abs().sum(2) + 1e-40
            assert bool(((dw.double() - parts.sum(2)).abs() <= bound).all())
            assert bool((dw[~held] == 0).all())


@pytest.mark.parametrize("K", (5, 64, 777, 4096))
def test_what_a_slot_without_a_place_does(K):
    """it reads no row, not even a NaN at place 0; its weight shows only where it is NaN; places outside of R are none"""
    R = torch.full((4, K), NAN, device="cuda")
    R[1], R[2] = 1.0, 2.0
    places = torch.tensor([[1, 2], [-1, 1], [-1, -1], [4, 2], [2, -2 ** 31], [2 ** 31 - 1, 1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[1.0, 1.0], [5.0, 1.0], [NAN, NAN], [3.0, 1.0], [1.0, 9.0], [1.0, 4.0]], device="cuda")
    out = torch.empty((6, K), device="cuda")
    G.groot_routed_sum(R, places, w, None, out)
    want = torch.tensor([3.0, 1.0, NAN, 2.0, 2.0, 4.0], device="cuda")[:, None].expand(6, K)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(out[~torch.isnan(out)], want[~torch.isnan(want)])
    G.groot_routed_sum(R, places, None, None, out)
    assert torch.equal(out, torch.tensor([3.0, 1.0, 0.0, 2.0, 2.0, 1.0], device="cuda")[:, None].expand(6, K))
    dR, dw = torch.full((4, K), 9.0, device="cuda"), torch.full((6, 2), 9.0, device="cuda")
    once = torch.tensor([[1, 2], [-1, -7], [-1, -1], [4, 0], [5, -2 ** 31], [2 ** 31 - 1, -1]], dtype=torch.int32, device="cuda")
    G.groot_routed_sum_backward(torch.full((6, K), INF, device="cuda"), R, once, w, dR, dw)
    assert bool((dw[1:3] == 0).all()) and float(dw[3, 0]) == 0 and bool((dw[4:] == 0).all()) and bool((dR[3] == 9).all()) and bool((dR[:3] == INF).all())
    X = torch.arange(6.0, device="cuda")[:, None].expand(6, K).contiguous()
    dR.fill_(9.0)
    G.groot_routed_rows(X, once, dR)
    assert torch.equal(dR[:, 0], torch.tensor([3.0, 0.0, 0.0, 9.0], device="cuda"))


def test_rows_behind_two_gigabytes():
    """offsets beyond 2^32 bytes: a matrix of 40,000 rows 32,768 columns apart (5.2 GB), and a stride of 2^31 bytes"""
    n, k, K, stride = 20000, 2, 48, 32768
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("not enough memory")
    places, m, gen = dealt(n, k, 8, 130, empty=0.1, spare=0)
    X = matrix(gen, n, K, torch.float32)
    R = torch.empty((m, stride), device="cuda")[:, 5:5 + K]
    G.groot_routed_rows(X, places, R)
    out = torch.empty_like(X)
    G.groot_routed_sum(R, places, None, None, out)
    count = (places >= 0).sum(1, keepdim=True)
    assert torch.equal(out, X * count)
    dR, dw = torch.empty((m, stride), device="cuda")[:, 1:1 + K], torch.empty((n, k), device="cuda")
    G.groot_routed_sum_backward(X, R, places, None, dR, dw)
    assert torch.equal(dR, R)
    far = torch.empty(3 * (1 << 29) + 64, device="cuda").as_strided((4, 8), (1 << 29, 1))
    x = torch.randn((4, 8), device="cuda")
    G.groot_routed_rows(x, torch.tensor([[3], [1], [0], [2]], dtype=torch.int32, device="cuda"), far)
    assert torch.equal(far, x[[2, 1, 3, 0]])


def test_no_rows_and_no_places():
    i = torch.zeros((0, 2), dtype=torch.int32, device="cuda")
    e = torch.empty((0, 16), device="cuda")
    R = torch.full((5, 16), 3.0, device="cuda")
    G.groot_routed_rows(e, i, R)
    G.groot_routed_sum(R, i, None, None, e)
    G.groot_routed_sum_backward(e, R, i, None, R.clone(), torch.empty((0, 2), device="cuda"))
    places = torch.full((4, 2), -1, dtype=torch.int32, device="cuda")
    X, out, dw = torch.ones((4, 16), device="cuda"), torch.full((4, 16), NAN, device="cuda"), torch.full((4, 2), NAN, device="cuda")
    G.groot_routed_rows(X, places, e)
    G.groot_routed_sum(e, places, None, X, out)
    G.groot_routed_sum_backward(X, e, places, None, None, dw)
    assert torch.equal(out, X) and bool((dw == 0).all()) and bool((R == 3).all())


# ---------------------------------------------------------------------------------------------------------------
# arguments, streams, graphs
# ---------------------------------------------------------------------------------------------------------------
def test_arguments_are_checked():
    x, i = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    w, off, R = torch.zeros((4, 2), device="cuda"), torch.zeros(9, dtype=torch.int64, device="cuda"), torch.zeros((8, 8), device="cuda")
    j = i.clone()
    for error, call in [
            (ValueError, lambda: G.groot_route(x, w[0], i, w, j, off, None)), (TypeError, lambda: G.groot_route(x, None, i.long(), w, j, off, None)),
            (TypeError, lambda: G.groot_route(x, None, i, w.half(), j, off, None)), (ValueError, lambda: G.groot_route(x, None, i, w, j, off[:8], None)),
            (TypeError, lambda: G.groot_route(x.double(), None, i, w, j, off, None)), (ValueError, lambda: G.groot_route(x.t(), None, i, w, j, off, None)),
            (G.GrootError, lambda: G.groot_route(x, None, i, w, j, off, None, sets=3)), (G.GrootError, lambda: G.groot_route(x, None, i, w, i, off, None)),
            (G.GrootError, lambda: G.groot_route(x, None, i, w, j, off, None, gate=5)), (ValueError, lambda: G.groot_route_backward(x, i, w, R)),
            (TypeError, lambda: G.groot_route_backward(x, i, w, x.half())), (TypeError, lambda: G.groot_routed_rows(x, i, R.half())),
            (ValueError, lambda: G.groot_routed_rows(x, i, R[:, :4])), (ValueError, lambda: G.groot_routed_rows(x, i, R, w[:, 0].contiguous())),
            (ValueError, lambda: G.groot_routed_rows(x, i[:3], R)), (TypeError, lambda: G.groot_routed_rows(x.double(), i, R.double())),
            (TypeError, lambda: G.groot_routed_sum(R, i, w, x.half(), x)), (G.GrootError, lambda: G.groot_routed_sum(R, i, w, x, x)),
            (ValueError, lambda: G.groot_routed_sum(R, i, w[:, :1].contiguous(), None, x)), (TypeError, lambda: G.groot_routed_sum(R, i, w.double(), None, x)),
            (ValueError, lambda: G.groot_routed_sum_backward(x, R, i, w, None, None)), (ValueError, lambda: G.groot_routed_sum_backward(x, None, i, w, R, w.clone())),
            (G.GrootError, lambda: G.groot_routed_sum_backward(x, R, i, w, R, w.clone())),
            (TypeError, lambda: G.groot_routed_sum_backward(x, R, i, w, R.half(), None))]:
        with pytest.raises(error):
            call()


def routed_step(t, ws):
    """one pass through all calls, on buffers that are there"""
    G.groot_route(t["scores"], t["bias"], t["experts"], t["weights"], t["places"], t["offsets"], ws, gate=G.GROOT_SIGMOID, sets=4, open_sets=2, set_best=2)
    G.groot_routed_rows(t["X"], t["places"], t["R"])
    G.groot_routed_sum(t["R"], t["places"], t["weights"], t["X"], t["out"])
    G.groot_routed_sum_backward(t["dout"], t["R"], t["places"], t["weights"], t["dR"], t["dw"])
    G.groot_routed_sum(t["dR"], t["places"], None, None, t["dX"])
    G.groot_route_backward(t["scores"], t["experts"], t["dw"], t["ds"], gate=G.GROOT_SIGMOID)
    return [t[k] for k in ("experts", "weights", "places", "offsets", "R", "out", "dR", "dw", "dX", "ds")]


def step_tensors(n, E, k, K, seed):
    scores, bias = made(n, E, torch.bfloat16, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X, dout = matrix(gen, n, K, torch.bfloat16), matrix(gen, n, K, torch.bfloat16)
    e, w, p, o = buffers(n, E, k)
    zeros = lambda *s, type=torch.bfloat16: torch.zeros(s, dtype=type, device="cuda")  # noqa: E731
    return dict(scores=scores, bias=bias, X=X, dout=dout, experts=e, weights=w, places=p, offsets=o, R=zeros(n * k, K), dR=zeros(n * k, K), out=zeros(n, K), dX=zeros(n, K),
                dw=zeros(n, k, type=torch.float32), ds=zeros(n, E))


@pytest.mark.parametrize("n", (3, 700, 20000))
def test_calls_run_under_graph_capture(n):
    """captured once, replayed on fresh inputs with eager work between: every replay is what the eager calls give"""
    E, k, K = 32, 4, 72
    t = step_tensors(n, E, k, K, 140)
    ws = workspace(G.groot_route_workspace(n, E, k))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        routed_step(t, ws)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = routed_step(t, ws)
    for seed in (141, 142, 143):
        fresh = step_tensors(n, E, k, K, seed)
        want = [x.clone() for x in routed_step(fresh, workspace(G.groot_route_workspace(n, E, k)))]
        for name in ("scores", "bias", "X", "dout"):
            t[name].copy_(fresh[name])
        for x in outs:
            x.zero_()
        ws.fill_(0x33)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_another_stream_and_the_same_bits():
    t = step_tensors(5000, 64, 8, 200, 150)
    ws = workspace(G.groot_route_workspace(5000, 64, 8))
    want = [x.clone() for x in routed_step(t, ws)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    e, w, p, o = buffers(5000, 64, 8)
    R = torch.zeros_like(t["R"])
    side.wait_stream(torch.cuda.current_stream())
    G.groot_route(t["scores"], t["bias"], e, w, p, o, ws, gate=G.GROOT_SIGMOID, sets=4, open_sets=2, set_best=2, stream=side)
    G.groot_routed_rows(t["X"], p, R, stream=side)
    side.synchronize()
    assert torch.equal(e, want[0]) and torch.equal(w, want[1]) and torch.equal(p, want[2]) and torch.equal(R, want[4])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(routed_step(t, ws), want))
