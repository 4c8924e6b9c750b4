"""The root-mean-square norm, its output in 8 bits and its gradients, against plain implementations.

Every operation of the forward call is rounded by itself, so Y, Q and the scales have to be equal to what the stated operations give: those are
done one by one by torch, in fp32 where the call is, with the sum of the squares in 64 bits.  (Its order could move a sum by 2^-53 of itself per
addition, which moves the rounding of rstd in one row of 10^7; a second check against 64 bits allows three roundings of fp32 and one of the type.)
Gradients, u = 2^-24: dX = rstd (a - h rstd^2 c) + dH: a is rounded once, c = mean of a h (K products, each rounded with the sums of the four or eight of a
lane in fp32, the rest in 64 bits: 10 u of the terms' magnitudes), five more operations: 16 u of the terms' magnitudes and one rounding to the type.
dgain: a term is rounded three times, and a group of lanes adds the terms of its rows in fp32, at most n / 512 + 16 of them here: (rows + 4) u, one rounding.
"""
import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")
EPS = 1e-6


def matrix(gen, rows, cols, dtype, pad=0, scale=1.0):
    wide = torch.randn((max(rows, 1), cols + pad), generator=gen, device="cuda") * scale
    return wide.to(dtype)[:rows, pad // 2:pad // 2 + cols]


def guarded(rows, cols, dtype, pad=0):
    wide = torch.full((max(rows, 1), cols + pad), 77, device="cuda").to(dtype)
    return wide[:rows, pad // 2:pad // 2 + cols], wide


def untouched(wide, view, pad):
    cols = view.shape[1]
    return bool((wide[:, :pad // 2] == 77).all() and (wide[:, pad // 2 + cols:] == 77).all())


def plain(X, residual, gain, eps=EPS):
    """h, rstd, y in fp32 and the codes with their scales, operation by operation"""
    T = X.dtype
    h = X.float() if residual is None else (X.float() + residual.float()).to(T).float()
    rstd = (1 / torch.sqrt(h.double().square().sum(1) / X.shape[1] + eps)).float()
    y = h * rstd[:, None]
    y = y if gain is None else y * gain.float()
    scale = y.abs().amax(1) * torch.tensor(1 / 127, dtype=torch.float32, device="cuda")
    scale = torch.where(torch.isfinite(y).all(1), scale, torch.full_like(scale, NAN))
    q = torch.where(scale[:, None] > 0, torch.round(y / scale[:, None]), torch.zeros_like(y)).to(torch.int8)
    return h, rstd, y, q, scale


# rows, width, columns beside
SHAPES = [(1, 1, 0), (3, 2, 1), (5, 3, 0), (7, 4, 4), (9, 7, 1), (33, 8, 0), (20, 9, 3), (100, 16, 0), (65, 31, 1), (40, 64, 0), (1000, 64, 8), (17, 65, 7), (50, 100, 4), (31, 127, 1),
          (12, 128, 0), (30, 129, 0), (21, 255, 3), (10, 256, 8), (6, 500, 0), (1, 512, 0), (8, 777, 1), (5, 1023, 0), (9, 1024, 16), (4, 2047, 1), (70, 2048, 0), (3, 2049, 3),
          (1, 4096, 0), (300, 4096, 8), (3, 4099, 1), (2, 8191, 0), (5, 8192, 0), (2, 8200, 8), (3, 16385, 3), (2, 32768, 0), (2, 40001, 1), (2, 65535, 1), (3, 65536, 0)]


def same(a, b, what):
    assert torch.equal(torch.isnan(a), torch.isnan(b)), what
    bad = (a != b) & ~torch.isnan(a)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}: {a[bad][0]} for {b[bad][0]}"


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(SHAPES)))
@pytest.mark.parametrize("stream", (False, True))
def test_norm(kind, case, stream):
    n, K, pad = SHAPES[case]
    T = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(200 + case)
    X, residual = matrix(gen, n, K, T, pad), matrix(gen, n, K, T, 2 * pad, 3.0) if stream else None
    gain = (1 + 0.2 * torch.randn(K, generator=gen, device="cuda")).to(T) if case % 3 else None
    Y, wide = guarded(n, K, T, pad)
    H, wide_h = guarded(n, K, T, 2 * pad)
    Q, wide_q = guarded(n, K, torch.int8, pad)
    scale, rstd = torch.full((n,), NAN, device="cuda"), torch.full((n,), NAN, device="cuda")
    G.groot_rms_norm(X, residual, gain, EPS, Y, H=H, Q=Q, q_scale=scale, rstd=rstd)
    h, r, y, q, s = plain(X, residual, gain)
    same(H.float(), h, "H")
    same(rstd, r, "rstd")
    same(Y.float(), y.to(T).float(), "Y")
    same(scale, s, "scale")
    same(Q, q, "Q")
    assert untouched(wide, Y, pad) and untouched(wide_h, H, 2 * pad) and untouched(wide_q, Q, pad)
    h = h.double()
    want = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * (1.0 if gain is None else gain.double())
    assert bool(((Y.double() - want).abs() <= (3 * U + 1.01 * UNIT[T]) * want.abs() + LEAST[T]).all())
    # each output by itself, and the same cut from the rows in the call of its own where they are in fp32
    alone = torch.full_like(Y, NAN)
    G.groot_rms_norm(X, residual, gain, EPS, alone)
    same(alone.float(), Y.float(), "Y alone")
    q2, s2 = torch.zeros_like(Q).contiguous(), torch.zeros_like(scale)
    G.groot_rms_norm(X, residual, gain, EPS, None, Q=q2, q_scale=s2)
    same(q2, Q, "Q alone")
    if T == torch.float32:
        G.groot_quantize_rows(Y, q2, s2)
        same(q2, Q, "groot_quantize_rows")
        same(s2, scale, "groot_quantize_rows")
    if stream:                                             # a stream that is updated in place
        held = residual.clone()
        x = X.clone()
        G.groot_rms_norm(x, held, gain, EPS, x, H=held)
        same(held.float(), H.float(), "H in place")
        same(x.float(), Y.float(), "Y in place")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("K", (5, 64, 1000, 4096))
def test_special_rows(kind, K):
    T = TYPES[kind]
    top = torch.finfo(T).max
    X = torch.randn((9, K), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(T)
    X[1] = 0
    X[2, K // 2] = NAN
    X[3, K - 1] = INF
    X[4] = top
    X[5] = torch.finfo(T).tiny
    X[6] = 0
    X[6, K - 1] = top
    X[7] = -1.0
    gain = torch.ones(K, device="cuda").to(T)
    gain[0] = 3.0
    Y, Q = torch.zeros_like(X), torch.zeros((9, K), dtype=torch.int8, device="cuda")
    scale, rstd = torch.zeros(9, device="cuda"), torch.zeros(9, device="cuda")
    G.groot_rms_norm(X, None, gain, EPS, Y, Q=Q, q_scale=scale, rstd=rstd)
    h, r, y, q, s = plain(X, None, gain)
    same(rstd, r, "rstd")
    same(Y.float(), y.to(T).float(), "Y")
    same(scale, s, "scale")
    same(Q, q, "Q")
    assert bool((Q[1] == 0).all() and (Q[2] == 0).all() and (Q[3] == 0).all()) and float(scale[1]) == 0 and bool(torch.isnan(scale[2:4]).all())
    assert bool((Q[8].abs().max() == 127).all()) and bool(torch.isfinite(Y[4].float()).all())


@pytest.mark.parametrize("eps", (1e-12, 1.0, 1e30))
def test_eps(eps):
    X = torch.randn((6, 96), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda") * 1e-4
    Y = torch.empty_like(X)
    G.groot_rms_norm(X, None, None, eps, Y)
    same(Y, plain(X, None, None, eps)[2], "Y")


def backward64(h, gain, dY, dH, eps=EPS):
    h, dY = h.double(), dY.double()
    g = torch.ones(h.shape[1], dtype=torch.float64, device="cuda") if gain is None else gain.double()
    rstd = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    a = dY * g
    c = (a * h).mean(1, keepdim=True)
    dX = rstd * (a - h * rstd ** 2 * c) + (0 if dH is None else dH.double())
    terms = rstd * (a.abs() + h.abs() * rstd ** 2 * (a * h).abs().mean(1, keepdim=True)) + (0 if dH is None else dH.double().abs())
    return dX, terms, (dY * h * rstd).sum(0), (dY * h * rstd).abs().sum(0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_backward(kind, case):
    n, K, pad = SHAPES[case]
    T = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(300 + case)
    H, dY, dH = matrix(gen, n, K, T, pad, 2.0), matrix(gen, n, K, T, 2 * pad), matrix(gen, n, K, T, pad) if case % 2 else None
    gain = (1 + 0.2 * torch.randn(K, generator=gen, device="cuda")).to(T) if case % 3 else None
    rstd, Y = torch.empty(n, device="cuda"), torch.empty((n, K), device="cuda", dtype=T)
    G.groot_rms_norm(H, None, gain, EPS, Y, rstd=rstd)
    dX, wide = guarded(n, K, T, pad)
    want, terms, want_gain, gain_terms = backward64(H, gain, dY, dH)
    for gtype in {T, torch.float32}:
        dgain = torch.full((K,), NAN, device="cuda").to(gtype)
        work = torch.full((max(16, G.groot_rms_norm_backward_workspace(n, K, T)),), 0x5A, dtype=torch.uint8, device="cuda")
        G.groot_rms_norm_backward(H, rstd, gain, dY, dX, dgain, work, dH=dH)
        err = (dX.double() - want).abs()
        bound = 16 * U * terms + 1.01 * UNIT[T] * want.abs() + LEAST[T]
        assert bool((err <= bound).all()), (err / bound).max()
        err = (dgain.double() - want_gain).abs()
        bound = (n / 512 + 20) * U * gain_terms + 1.01 * UNIT[gtype] * want_gain.abs() + LEAST[gtype]
        assert bool((err <= bound).all()), (err / bound).max()
    assert untouched(wide, dX, pad)
    kept = dX.clone()
    G.groot_rms_norm_backward(H, rstd, gain, dY, dX, None, None, dH=dH)
    assert torch.equal(kept, dX)


@pytest.mark.parametrize("n, K", ((20000, 64), (3000, 1000), (9000, 33), (4000, 4096)))
def test_gain_gradient_of_many_rows(n, K):
    """exact: terms of whole numbers, whose sums fp32 holds, lose no row"""
    gen = torch.Generator(device="cuda").manual_seed(7)
    H = torch.randint(-2, 3, (n, K), generator=gen, device="cuda").float()
    dY = torch.randint(-1, 2, (n, K), generator=gen, device="cuda").float()
    rstd = torch.ones(n, device="cuda")
    dX, dgain = torch.empty_like(H), torch.empty(K, device="cuda")
    work = torch.empty(G.groot_rms_norm_backward_workspace(n, K, torch.float32), dtype=torch.uint8, device="cuda")
    G.groot_rms_norm_backward(H, rstd, None, dY, dX, dgain, work)
    assert torch.equal(dgain.double(), (H.double() * dY.double()).sum(0))


def test_backward_by_differences():
    """the loss sum(Y w) + sum(H v) moves along a direction by the gradient, to second order (differences of both sides in 64 bits)"""
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, K, step = 40, 96, 1e-4
    x, w, v, along = (torch.randn((n, K), generator=gen, device="cuda") for _ in range(4))
    gain, along_g = torch.rand(K, generator=gen, device="cuda") + 0.5, torch.randn(K, generator=gen, device="cuda")

    def loss(t):
        h, g = x.double() + t * along.double(), gain.double() + t * along_g.double()
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * g
        return (y * w.double() + h * v.double()).sum()
    rstd, Y, dX, dgain = torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty_like(x), torch.empty_like(gain)
    G.groot_rms_norm(x, None, gain, EPS, Y, rstd=rstd)
    G.groot_rms_norm_backward(x, rstd, gain, w, dX, dgain, torch.empty(G.groot_rms_norm_backward_workspace(n, K, x.dtype), dtype=torch.uint8, device="cuda"), dH=v)
    got = (dX.double() * along.double()).sum() + (dgain.double() * along_g.double()).sum()
    want = (loss(step) - loss(-step)) / (2 * step)
    # third derivatives of 3840 terms of size 1 to 10 times step^2 / 6, and fp32's rounding of as many terms
    assert abs(float(got - want)) <= 3840 * 10 * step ** 2 + 3840 * 16 * U * 10


def test_no_rows():
    x = torch.empty((0, 64), device="cuda")
    G.groot_rms_norm(x, None, None, EPS, x.clone())
    dgain = torch.full((64,), NAN, device="cuda")
    G.groot_rms_norm_backward(x, torch.empty(0, device="cuda"), None, x, x.clone(), dgain, torch.empty(max(16, G.groot_rms_norm_backward_workspace(0, 64, x.dtype)), dtype=torch.uint8, device="cuda"))
    assert bool((dgain == 0).all())


def test_rows_behind_two_gigabytes():
    """offsets beyond 2^32 bytes"""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    n, K, stride = 30000, 40, 65536
    X = torch.empty((n, stride), device="cuda", dtype=torch.bfloat16)[:, 3:3 + K]
    X.copy_(torch.randn((n, K), generator=torch.Generator(device="cuda").manual_seed(9), device="cuda"))
    Y = torch.empty((n, stride), device="cuda", dtype=torch.bfloat16)[:, 1:1 + K]
    rstd = torch.empty(n, device="cuda")
    G.groot_rms_norm(X, None, None, EPS, Y, rstd=rstd)
    want = plain(X.contiguous(), None, None)
    same(Y.float(), want[2].to(X.dtype).float(), "Y")
    dX, near = torch.empty((n, stride), device="cuda", dtype=torch.bfloat16)[:, 5:5 + K], torch.empty((n, K), device="cuda", dtype=torch.bfloat16)
    G.groot_rms_norm_backward(X, rstd, None, Y, dX, None, None)
    G.groot_rms_norm_backward(X.contiguous(), rstd, None, Y.contiguous(), near, None, None)
    assert torch.equal(dX, near)


def test_arguments_are_checked():
    x, g, r = torch.zeros((4, 64), device="cuda"), torch.ones(64, device="cuda"), torch.zeros(4, device="cuda")
    y, q = torch.zeros_like(x), torch.zeros((4, 64), dtype=torch.int8, device="cuda")
    for error, call in [
            (TypeError, lambda: G.groot_rms_norm(x.double(), None, None, EPS, y)), (TypeError, lambda: G.groot_rms_norm(x, x.half(), None, EPS, y)),
            (ValueError, lambda: G.groot_rms_norm(x, x[:3], None, EPS, y)), (ValueError, lambda: G.groot_rms_norm(x, None, g[:63], EPS, y)),
            (TypeError, lambda: G.groot_rms_norm(x, None, g.half(), EPS, y)), (TypeError, lambda: G.groot_rms_norm(x, None, g, EPS, y.half())),
            (ValueError, lambda: G.groot_rms_norm(x.t(), None, None, EPS, y.t())), (G.GrootError, lambda: G.groot_rms_norm(x, None, g, 0.0, y)),
            (G.GrootError, lambda: G.groot_rms_norm(x, None, g, EPS, None)), (G.GrootError, lambda: G.groot_rms_norm(x, None, g, EPS, y, Q=q)),
            (TypeError, lambda: G.groot_rms_norm(x, None, g, EPS, y, Q=x, q_scale=r)), (ValueError, lambda: G.groot_rms_norm(x, None, g, EPS, y, rstd=r[:3])),
            (G.GrootError, lambda: G.groot_rms_norm(x[:3], None, g, EPS, x[1:])), (G.GrootError, lambda: G.groot_rms_norm(x, y, g, EPS, x, H=x)),
            (G.GrootError, lambda: G.groot_rms_norm_backward(x, r, g, y, x, None, None)), (G.GrootError, lambda: G.groot_rms_norm_backward(x, r, g, y, x.clone(), g.clone(), None)),
            (TypeError, lambda: G.groot_rms_norm_backward(x, r, g, y.half(), x.clone(), None, None)), (TypeError, lambda: G.groot_rms_norm_backward(x, r.double(), g, y, x.clone(), None, None)),
            (G.GrootError, lambda: G.groot_rms_norm_backward(x.half(), r, None, y.half(), x.half(), g.bfloat16(), torch.empty(1 << 20, device="cuda")))]:
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("n, K, T", ((1, 4096, torch.bfloat16), (5000, 64, torch.float32), (300, 8193, torch.float16)))
def test_calls_run_under_graph_capture(n, K, T):
    gen = torch.Generator(device="cuda").manual_seed(10)
    t = {name: matrix(gen, n, K, T) for name in ("X", "residual", "dY", "dH")}
    t["gain"] = torch.randn(K, generator=gen, device="cuda").to(T)
    H, Y, dX = (torch.zeros_like(t["X"]) for _ in range(3))
    dgain = torch.zeros_like(t["gain"])
    Q, scale, rstd = torch.zeros((n, K), dtype=torch.int8, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    work = torch.empty(max(16, G.groot_rms_norm_backward_workspace(n, K, T)), dtype=torch.uint8, device="cuda")
    outs = [H, Y, Q, scale, rstd, dX, dgain]

    def step():
        G.groot_rms_norm(t["X"], t["residual"], t["gain"], EPS, Y, H=H, Q=Q, q_scale=scale, rstd=rstd)
        G.groot_rms_norm_backward(H, rstd, t["gain"], t["dY"], dX, dgain, work, dH=t["dH"])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for x in t.values():
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        step()
        want = [x.clone() for x in outs]
        for x in outs:
            x.zero_()
        work.fill_(0x33)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
