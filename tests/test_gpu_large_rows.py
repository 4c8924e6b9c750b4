"""Routed rows, their sums and gradients, and the norm on matrices that no cache holds: those kernels load and store past the caches.

Every number of lanes and pieces that a row can get, whole rows and rows that begin and end anywhere, against plain implementations in 64 bits; also
the gradients of a thousand to two thousand wide rows, whose workgroups walk through all slots of a row.  Tolerances as for small matrices, from the
arithmetic that the calls state (u = 2^-24, half a step of fp32):
  * sum: k products and additions: (k + 2) 2 u of the terms' magnitudes and one rounding to the type; its gradients: one product and a rounding, and
    for the weights K terms, (K + 2) 2 u of their magnitudes.
  * norm: Y three roundings of fp32 and one of the type; dX 16 u of its terms' magnitudes and one rounding (the product of two values, the sum of a
    lane's 4 or 8 of them, five more operations); dgain: a term is rounded three times, and the rows of a group of lanes add up in fp32.  At least 256
    workgroups take the rows, so these are at most n / 256 + 1.
"""
import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402
from test_gpu_norm import EPS, backward64, plain  # noqa: E402
from test_gpu_routed import LEAST, TYPES, U2, UNIT, dealt, guarded, matrix, slots64, untouched  # noqa: E402

pytestmark = pytest.mark.gpu

U, NAN, INF = 2.0 ** -24, float("nan"), float("inf")
LARGE = 264 << 20                                          # bytes


def width(pieces, odd, size):
    """columns of a row of so many 16 bytes; odd: one less"""
    return pieces * 16 // size - odd


def rows_for(K, size, copies=1):
    return LARGE // (K * size * copies) + 1


def check(got, want, bound, what):
    for i in range(0, got.shape[0], 1 << 20):               # in 64 bits, a part at a time
        g, w, b = (t[i:i + (1 << 20)] for t in (got, want, bound))
        bad = ~((g.double() - w).abs() <= b)
        assert not bad.any(), f"{what}: {int(bad.sum())} off in rows from {i} on, first at {bad.nonzero()[0].tolist()}: {g[bad][0]} for {w[bad][0]}"


# pieces of a row, columns less: one width for every number of lanes and pieces in a lane
WIDTHS = [(1, 1), (9, 0), (16, 1), (40, 0), (64, 1), (128, 0), (127, 1), (256, 0), (250, 1), (512, 0), (700, 1), (1100, 1)]


@pytest.mark.parametrize("kind", list(TYPES) + ["i8"])
@pytest.mark.parametrize("pieces, odd", WIDTHS)
def test_rows_to_their_places(kind, pieces, odd):
    dtype = TYPES.get(kind, torch.int8)
    size, k, pad = dtype.itemsize, 2, 3 * odd
    K = width(pieces, odd, size)
    n = rows_for(K, size, k)
    places, m, gen = dealt(n, k, 5, 160 + pieces, empty=0.01)
    X = matrix(gen, n, K, dtype, pad)
    R, wide = guarded(m, K, dtype, pad)
    G.groot_routed_rows(X, places, R)
    i, s = torch.nonzero(places >= 0, as_tuple=True)
    want = torch.full((m, K), 77.0, device="cuda").to(dtype)
    want[places[i, s].long()] = X[i]
    assert torch.equal(R, want) and untouched(wide, R, pad)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("pieces, odd", WIDTHS)
def test_sum_over_the_places(kind, pieces, odd):
    dtype, k, pad = TYPES[kind], 2, 3 * odd
    K = width(pieces, odd, dtype.itemsize)
    n = rows_for(K, dtype.itemsize)
    places, m, gen = dealt(n, k, 5, 180 + pieces)
    R = matrix(gen, m, K, dtype, pad)
    R[m - 3:] = NAN                                         # behind the last place
    w, addend = torch.randn((n, k), generator=gen, device="cuda"), matrix(gen, n, K, dtype, 2 * pad)
    out, wide = guarded(n, K, dtype, pad)
    G.groot_routed_sum(R, places, w, addend, out)
    parts = slots64(R, places) * w.double()[:, :, None]
    want, terms = addend.double() + parts.sum(1), addend.double().abs() + parts.abs().sum(1)
    check(out, want, (k + 2) * U2 * terms + UNIT[dtype] * want.abs() * 1.01 + LEAST[dtype], "sum")
    assert untouched(wide, out, pad)


def check_sum_backward(dtype, n, k, E, K, pad, seed):
    places, m, gen = dealt(n, k, E, seed)
    R, dout = matrix(gen, m, K, dtype, pad), matrix(gen, n, K, dtype, 2 * pad)
    w = torch.randn((n, k), generator=gen, device="cuda")
    dR, wide = guarded(m, K, dtype, pad)
    dw = torch.full((n, k), NAN, device="cuda")
    G.groot_routed_sum_backward(dout, R, places, w, dR, dw)
    for slot in range(k):                                   # a slot at a time: 64 bits of all would take much memory
        held = places[:, slot] >= 0
        at, rows = places[held, slot].long(), dout[held].double()
        want = rows * w[held, slot, None].double()
        check(dR[at], want, 2 * U2 * want.abs() + UNIT[dtype] * want.abs() * 1.01 + LEAST[dtype], f"dR, slot {slot}")
        terms = R[at].double() * rows
        check(dw[held, slot], terms.sum(1), (K + 2) * U2 * terms.abs().sum(1) + 1e-40, f"dweights, slot {slot}")
    assert bool((dw[places < 0] == 0).all()) and bool((dR[m - 3:] == torch.tensor(77.0).to(dtype)).all()) and untouched(wide, dR, pad)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("pieces, odd", WIDTHS)
def test_sum_backward(kind, pieces, odd):
    dtype = TYPES[kind]
    K = width(pieces, odd, dtype.itemsize)
    check_sum_backward(dtype, rows_for(K, dtype.itemsize, 3), 3, 5, K, 3 * odd, 200 + pieces)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("pieces, odd", [(256, 0), (256, 1)])
def test_sum_backward_of_many_slots(kind, pieces, odd):
    """fewer than 2048 rows, a workgroup each"""
    dtype = TYPES[kind]
    check_sum_backward(dtype, 2047, 32, 40, width(pieces, odd, dtype.itemsize), 3 * odd, 215)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n, pieces, odd", [(1024, 200, 0), (1500, 300, 1), (2047, 256, 0), (2048, 255, 1), (2100, 700, 0), (1100, 1100, 1), (1025, 90, 1)])
def test_sum_backward_of_some_wide_rows(kind, n, pieces, odd):
    dtype = TYPES[kind]
    check_sum_backward(dtype, n, 5, 9, width(pieces, odd, dtype.itemsize), 3 * odd, 220 + pieces)


NORM_WIDTHS = [(1, 1), (16, 0), (31, 1), (64, 0), (127, 1), (192, 1), (256, 0), (383, 1), (512, 0), (768, 1), (1024, 0), (2000, 1), (4096, 0), (8000, 1), (16384, 1)]


@pytest.mark.parametrize("kind, pieces, odd", [(kind, p, odd) for p, odd in NORM_WIDTHS for kind in TYPES if width(p, odd, TYPES[kind].itemsize) <= 65536])
def test_norm_and_its_gradients(kind, pieces, odd):
    T, pad = TYPES[kind], 3 * odd
    K = width(pieces, odd, T.itemsize)
    n = rows_for(K, T.itemsize)
    gen = torch.Generator(device="cuda").manual_seed(240 + pieces)
    X, residual = matrix(gen, n, K, T, pad), matrix(gen, n, K, T, 2 * pad, 3.0)
    gain = (1 + 0.2 * torch.randn(K, generator=gen, device="cuda")).to(T)
    (H, wide_h), (Y, wide), (Q, wide_q) = guarded(n, K, T, 2 * pad), guarded(n, K, T, pad), guarded(n, K, torch.int8, pad)
    scale, rstd = torch.full((n,), NAN, device="cuda"), torch.full((n,), NAN, device="cuda")
    G.groot_rms_norm(X, residual, gain, EPS, Y, H=H, Q=Q, q_scale=scale, rstd=rstd)
    h, r, y, q, s = plain(X, residual, gain)
    assert torch.equal(H, h.to(T))
    # a sum of 65536 squares in 64 bits, 64 to a lane, is off by 2^-46 of itself at the most: rows whose rstd comes that close to the border between
    # two numbers of fp32 may be rounded either way (one in a million)
    exact = 1 / torch.sqrt(h.double().square().mean(1) + EPS)
    other = torch.nextafter(r, torch.where(exact > r, torch.full_like(r, INF), torch.zeros_like(r))).double()
    sure = (exact - (r.double() + other) / 2).abs() > 2.0 ** -44 * exact
    assert float(sure.double().mean()) > 0.999
    for name, a, b in (("rstd", rstd, r), ("Y", Y, y.to(T)), ("scale", scale, s), ("Q", Q, q)):
        a, b = a[sure], b[sure]
        assert torch.equal(a, b), f"{name}: {int((a != b).sum())} of {a.numel()} differ"
    assert untouched(wide_h, H, 2 * pad) and untouched(wide, Y, pad) and untouched(wide_q, Q, pad)
    del h, r, y, q, s, a, b, Y, wide, Q, wide_q, X, residual

    dY, dH = matrix(gen, n, K, T, 2 * pad), matrix(gen, n, K, T, pad)
    dX, wide = guarded(n, K, T, pad)
    dgain = torch.full((K,), NAN, device="cuda")
    work = torch.full((G.groot_rms_norm_backward_workspace(n, K, T),), 0x5A, dtype=torch.uint8, device="cuda")
    G.groot_rms_norm_backward(H, rstd, gain, dY, dX, dgain, work, dH=dH)
    want, terms, want_gain, gain_terms = backward64(H, gain, dY, dH)
    check(dX, want, 16 * U * terms + 1.01 * UNIT[T] * want.abs() + LEAST[T], "dX")
    check(dgain, want_gain, (n / 256 + 5) * U * gain_terms + 1.01 * U * want_gain.abs() + LEAST[torch.float32], "dgain")
    assert untouched(wide, dX, pad)

    # whole numbers, whose sums fp32 holds: no row is lost, and none counts twice
    H.copy_(torch.randint(-2, 3, (n, K), generator=gen, device="cuda", dtype=torch.int8))
    dY.copy_(torch.randint(-1, 2, (n, K), generator=gen, device="cuda", dtype=torch.int8))
    G.groot_rms_norm_backward(H, torch.ones_like(rstd), None, dY, dX, dgain, work)
    assert torch.equal(dgain.double(), (H * dY).sum(0, dtype=torch.float64))


def test_routing_more_rows_than_a_launch_of_256_lanes_a_workgroup_holds():
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("not enough memory")
    n = (1 << 30) + 70
    scores = torch.randint(0, 3, (n, 2), device="cuda", dtype=torch.int8, generator=torch.Generator(device="cuda").manual_seed(260)).half()
    experts, places = (torch.full((n, 1), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    weights, offsets = torch.full((n, 1), NAN, device="cuda"), torch.full((3,), -7, dtype=torch.int64, device="cuda")
    work = torch.empty(G.groot_route_workspace(n, 2, 1), dtype=torch.uint8, device="cuda")
    G.groot_route(scores, None, experts, weights, places, offsets, work)
    second = scores[:, 1] > scores[:, 0]                     # ties go to the first
    assert torch.equal(experts[:, 0], second.int()) and bool((weights == 1).all())
    upto = torch.cumsum(second, 0, dtype=torch.int32)
    firsts = n - int(upto[-1])
    assert offsets.tolist() == [0, firsts, n]
    for i in range(0, n, 1 << 26):
        u, s = upto[i:i + (1 << 26)], second[i:i + (1 << 26)]
        row = torch.arange(i, i + len(u), dtype=torch.int32, device="cuda")
        assert torch.equal(places[i:i + (1 << 26), 0], torch.where(s, firsts + u - 1, row - u)), i
