"""Grouped products, products in 8-bit integers and the AdamW step against plain implementations in 64 bits.

Tolerances, all derived from the arithmetic that the calls state:
  * sums of K products in 32 bits, in any order: every addition loses at most 2^-23 of a partial sum (half of that where it rounds
    to nearest), a product of fp32 values as much; 16-bit products are exact.  (K + 3) 2^-23 of the sum of the terms' magnitudes.
  * one rounding to the output's type: 2^-24, 2^-8 (bfloat16: 8 significant bits) or 2^-11 (float16) of the value, 2^-25 at least for float16.
  * 8-bit products: the integer sum is exact; its conversion, two products and a sum round once each.
"""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def rounding(y, dtype):
    return UNIT[dtype] * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133 if dtype == torch.bfloat16 else 1e-45)


def sum_bound(terms, K):
    return (K + 3) * 2.0 ** -23 * terms


def close(got, want, bound, what):
    assert torch.isfinite(got).all(), f"{what}: not finite (a value was not written?)"
    err = (got.double() - want).abs()
    bad = err > bound
    assert int(bad.sum()) == 0, f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}, worst {(err / bound.clamp(min=1e-300)).max():.3g} x"


def matrix(gen, rows, cols, dtype, pad=0, scale=1.0):
    """rows x cols inside a wider matrix (pad more columns, beginning at the pad's half)"""
    wide = torch.randn((max(rows, 1), cols + pad), generator=gen, device="cuda") * scale
    return wide.to(dtype)[:rows, pad // 2:pad // 2 + cols]


def out_matrix(rows, cols, dtype, pad=0):
    return torch.full((max(rows, 1), cols + pad), float("nan"), device="cuda").to(dtype)[:rows, pad // 2:pad // 2 + cols]


def offsets_of(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int64, device="cuda")


def group_of(sizes):
    return torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(sizes, device="cuda"))


# sizes of the groups, K, N, pad of the rows
SHAPES = [
    ([1], 64, 64, 0),
    ([1], 1, 1, 0),
    ([3, 0, 5, 1], 7, 3, 0),
    ([0, 0, 0], 32, 32, 0),
    ([64, 7840, 64], 32, 32, 0),
    ([64, 3000, 65], 64, 5, 0),
    ([700], 4, 32, 4),
    ([1, 2, 3, 0, 17, 31, 32, 33, 63, 64, 65], 128, 256, 8),
    ([127, 129, 255, 257], 192, 136, 0),
    ([300, 1], 333, 129, 1),
    ([40, 0, 300], 511, 65, 3),
    ([2, 1, 0, 4, 3, 1, 1, 2], 1024, 512, 0),
    ([513], 96, 1000, 0),
    ([1100, 20], 520, 264, 8),
    ([16] * 70, 40, 24, 0),
    ([5] * 5 + [0] * 200 + [90], 72, 80, 0),
    ([40, 0, 5000, 1, 2100], 64, 48, 0),
    ([9000], 20, 12, 0),
]


def case_tensors(dtype, sizes, K, N, pad, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, E = sum(sizes), len(sizes)
    X, dY = matrix(gen, n, K, dtype, pad), matrix(gen, n, N, dtype, pad)
    W = (torch.randn((E, K, N), generator=gen, device="cuda") / math.sqrt(K)).to(dtype)
    b = torch.randn((E, N), generator=gen, device="cuda").to(dtype)
    return n, E, X, dY, W, b


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_grouped_product_and_its_gradients(kind, case):
    dtype, (sizes, K, N, pad) = TYPES[kind], SHAPES[case]
    n, E, X, dY, W, b = case_tensors(dtype, sizes, K, N, pad, 100 + case)
    offsets, g = offsets_of(sizes), group_of(sizes)
    X64, dY64, W64, b64 = X.double(), dY.double(), W.double(), b.double()

    for relu in (False, True):
        Y = out_matrix(n, N, dtype, pad)
        G.groot_grouped_product(X, W, offsets, b if not relu else None, relu, Y)
        bias = torch.zeros_like(b64) if relu else b64
        want = torch.cat([x @ w + c for x, w, c in zip(X64.split(sizes), W64, bias)])
        terms = torch.cat([x.abs() @ w.abs() + c.abs() for x, w, c in zip(X64.split(sizes), W64, bias)])
        want = want.clamp(min=0) if relu else want
        close(Y, want, sum_bound(terms, K + 1) + rounding(want, dtype) * 1.01, "Y")

    dX = out_matrix(n, K, dtype, pad)
    G.groot_grouped_product_backward_data(dY, W, offsets, dX)
    want = torch.cat([d @ w.t() for d, w in zip(dY64.split(sizes), W64)])
    terms = torch.cat([d.abs() @ w.abs().t() for d, w in zip(dY64.split(sizes), W64)])
    close(dX, want, sum_bound(terms, N) + rounding(want, dtype) * 1.01, "dX")

    work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(n, E, K, N, dtype)), dtype=torch.uint8, device="cuda")
    lens = torch.tensor(sizes, device="cuda", dtype=torch.float64)
    for grad in {dtype, torch.float32}:
        dW = torch.full((E, K, N), float("nan"), device="cuda").to(grad)
        db = torch.full((E, N), float("nan"), device="cuda").to(grad)
        work.fill_(255)
        G.groot_grouped_product_backward_weights(X, dY, offsets, dW, db, work)
        want = torch.stack([x.t() @ d for x, d in zip(X64.split(sizes), dY64.split(sizes))])
        terms = torch.stack([x.abs().t() @ d.abs() for x, d in zip(X64.split(sizes), dY64.split(sizes))])
        close(dW, want, sum_bound(terms, lens[:, None, None]) + rounding(want, grad) * 1.01, "dW")
        want = torch.stack([d.sum(0) for d in dY64.split(sizes)])
        terms = torch.stack([d.abs().sum(0) for d in dY64.split(sizes)])
        close(db, want, sum_bound(terms, lens[:, None]) + rounding(want, grad) * 1.01, "db")
        again = torch.full_like(dW, float("nan"))
        work.zero_()
        G.groot_grouped_product_backward_weights(X, dY, offsets, again, None, work)
        assert torch.equal(dW, again), "dW differs from call to call"


@pytest.mark.parametrize("kind", TYPES)
def test_grouped_product_gradients_against_differences(kind):
    """L = sum(C * Y) is linear in X and in W, so central differences are exact but for the rounding of Y."""
    dtype, sizes, K, N, h = TYPES[kind], [5, 0, 70, 33], 48, 40, 0.25
    n, E, X, C, W, b = case_tensors(dtype, sizes, K, N, 0, 5)
    offsets = offsets_of(sizes)
    dX, dW, db = torch.empty_like(X), torch.empty((E, K, N), device="cuda"), torch.empty((E, N), device="cuda")
    G.groot_grouped_product_backward_data(C, W, offsets, dX)
    work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(n, E, K, N, dtype)), dtype=torch.uint8, device="cuda")
    G.groot_grouped_product_backward_weights(X, C, offsets, dW, db, work)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)

    def loss(X, W, b):
        Y = torch.empty((n, N), dtype=dtype, device="cuda")
        G.groot_grouped_product(X.to(dtype).contiguous(), W.to(dtype).contiguous(), offsets, b.to(dtype), False, Y)
        absolute = torch.cat([x.abs() @ w.abs() + c.abs() for x, w, c in zip(X.double().split(sizes), W.double(), b.double())])
        bound = (C.double().abs() * (sum_bound(absolute, K + 1) + UNIT[dtype] * 1.01 * absolute)).sum()
        return (C.double() * Y.double()).sum(), bound
    for which, grad in (("X", dX), ("W", dW), ("b", db)):
        base = {"X": X, "W": W, "b": b}
        D = torch.randint(-1, 2, base[which].shape, generator=gen, device="cuda").to(torch.float32)
        # the moved points in the type itself: their true distance is what the difference is taken over
        up, down = (base[which].float() + h * D).to(dtype), (base[which].float() - h * D).to(dtype)
        (lu, bu), (ld, bd) = loss(**{**base, which: up}), loss(**{**base, which: down})
        slope = (grad.double() * (up.double() - down.double())).sum()
        terms = torch.cat([x.abs() @ w.abs().t() for x, w in zip(C.double().split(sizes), W.double())]) if which == "X" else \
            torch.stack([x.abs().t() @ d.abs() for x, d in zip(X.double().split(sizes), C.double().split(sizes))]) if which == "W" else \
            torch.stack([d.abs().sum(0) for d in C.double().split(sizes)])
        unit = UNIT[dtype] if which == "X" else UNIT[torch.float32]
        off = ((sum_bound(terms, n + N) + unit * 1.01 * terms) * (up.double() - down.double()).abs()).sum()
        assert (lu - ld - slope).abs() <= bu + bd + off, which


def test_grouped_product_without_offsets_and_rows_outside_groups():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    X, W = matrix(gen, 300, 64, torch.bfloat16), matrix(gen, 64, 96, torch.bfloat16, scale=0.1)[None].contiguous()
    Y, Z = out_matrix(300, 96, torch.bfloat16), out_matrix(300, 96, torch.bfloat16)
    G.groot_grouped_product(X, W, None, None, False, Y)
    G.groot_grouped_product(X, W, torch.tensor([0, 300], device="cuda"), None, False, Z)
    assert torch.equal(Y, Z)
    # rows before the first and behind the last group stay as they were; offsets outside the rows count as the nearer end
    three = W.expand(3, 64, 96).contiguous()
    for offsets, low, high in (([10, 20, 20, 290], 10, 290), ([-5, 20, 40, 4000], 0, 300), ([7, 100, 50, 200], 7, 200), ([500, 600, 700, 800], 300, 300),
                               ([-(1 << 62), 5, 5, 1 << 62], 0, 300)):
        Z = out_matrix(300, 96, torch.bfloat16)
        G.groot_grouped_product(X, three, torch.tensor(offsets, device="cuda"), None, False, Z)
        if offsets[1] <= offsets[2]:
            assert torch.equal(Z[low:high], Y[low:high])
        assert torch.isnan(Z[:low]).all() and torch.isnan(Z[high:]).all()
        dX, dW = out_matrix(300, 64, torch.bfloat16), torch.full((3, 64, 96), float("nan"), device="cuda")
        work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(300, 3, 64, 96, torch.bfloat16)), dtype=torch.uint8, device="cuda")
        G.groot_grouped_product_backward_data(Y, three, torch.tensor(offsets, device="cuda"), dX)
        G.groot_grouped_product_backward_weights(X, Y, torch.tensor(offsets, device="cuda"), dW, None, work)
        assert torch.isfinite(dW).all() and torch.isnan(dX[:low]).all() and torch.isnan(dX[high:]).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n, K", [(200, 128), (3, 128), (200, 77)])
def test_values_that_are_not_finite_stay_in_their_row(kind, n, K):
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    X, W = matrix(gen, n, K, dtype), matrix(gen, K, 64, dtype)[None].contiguous()
    X = X.contiguous()
    Y0, Y = out_matrix(n, 64, dtype), out_matrix(n, 64, dtype)
    G.groot_grouped_product(X, W, None, None, True, Y0)
    X[1, 5], X[2, K - 1] = float("nan"), float("inf")
    G.groot_grouped_product(X, W, None, None, True, Y)
    keep = [r for r in range(n) if r not in (1, 2)]
    assert torch.equal(Y[keep], Y0[keep])
    assert torch.isnan(Y[1]).all()
    want = torch.where(W[0, K - 1] > 0, float("inf"), torch.where(W[0, K - 1] < 0, 0.0, float("nan")))
    assert torch.equal(torch.nan_to_num(Y[2].float(), nan=-1, posinf=-2), torch.nan_to_num(want.float(), nan=-1, posinf=-2))
    # behind a group's end and the widths' ends lie such values too, and none reaches a result
    wide = torch.full((n + 64, K + 24), float("nan"), device="cuda").to(dtype)
    wide[:n, 8:8 + K] = torch.where(torch.isfinite(X), X, torch.ones_like(X))
    inner = wide[:n, 8:8 + K]
    offsets = torch.tensor([0, n - 1], device="cuda")
    a, c = out_matrix(n, 64, dtype), out_matrix(n, 64, dtype)
    G.groot_grouped_product(inner, W, offsets, None, False, a)
    G.groot_grouped_product(inner.contiguous(), W, offsets, None, False, c)
    assert torch.isfinite(a[:n - 1]).all() and torch.equal(a[:n - 1], c[:n - 1]) and torch.isnan(a[n - 1]).all()
    dW = torch.full((1, K, 64), float("nan"), device="cuda")
    work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(n, 1, K, 64, dtype)), dtype=torch.uint8, device="cuda")
    dy = torch.full((n + 64, 64 + 24), float("inf"), device="cuda").to(dtype)
    dy[:n - 1, 8:72] = 1
    G.groot_grouped_product_backward_weights(inner, dy[:n, 8:72], offsets, dW, None, work)
    assert torch.isfinite(dW).all()


def test_offsets_that_do_not_ascend_stay_in_bounds():
    """groups that overlap ask for more pieces than the rows have room for: nothing beyond the workspace or the outputs is written"""
    n, K, N = 5000, 64, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    X, dY = matrix(gen, n, K, torch.bfloat16), matrix(gen, n, N, torch.bfloat16)
    offsets = torch.tensor([0, n] * 20 + [0], device="cuda")
    need = G.groot_grouped_product_backward_weights_workspace(n, 40, K, N, torch.bfloat16)
    work = torch.full((need + 4096,), 7, dtype=torch.uint8, device="cuda")
    dW = torch.empty((40, K, N), device="cuda")
    G.groot_grouped_product_backward_weights(X, dY, offsets, dW, None, work)
    assert (work[need:] == 7).all()


# sizes at which the larger tiles and the kernels for many columns and few rows are taken: (sizes of the groups, K, N)
LARGE = [([8192], 72, 4096), ([4000, 100, 60], 136, 2100), ([2048], 264, 2048), ([900], 200, 1100), ([256], 640, 4096), ([33] * 8, 1024, 640),
         ([300], 3600, 3600), ([700] * 16, 520, 1032), ([1] * 20, 640, 2048), ([9, 16, 2], 1000, 2052), ([7], 300, 5000), ([20000], 64, 96),
         ([5, 11], 77, 131), ([2], 1001, 515), ([16], 33, 6), ([1, 0, 3], 5, 9), ([70, 300], 3, 70), ([600], 1003, 258)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(LARGE)))
def test_large_sizes(kind, case):
    dtype, (sizes, K, N) = TYPES[kind], LARGE[case]
    n, E, X, dY, W, b = case_tensors(dtype, sizes, K, N, 0, 300 + case)
    offsets = offsets_of(sizes) if E > 1 else None
    parts = lambda t: t.double().split(sizes)  # noqa: E731
    Y, dX = out_matrix(n, N, dtype), out_matrix(n, K, dtype)
    G.groot_grouped_product(X, W, offsets, b, False, Y)
    want = torch.cat([x @ w + c for x, w, c in zip(parts(X), W.double(), b.double())])
    terms = torch.cat([x.abs() @ w.abs() + c.abs() for x, w, c in zip(parts(X), W.double(), b.double())])
    close(Y, want, sum_bound(terms, K + 1) + rounding(want, dtype) * 1.01, "Y")
    G.groot_grouped_product_backward_data(dY, W, offsets, dX)
    want = torch.cat([d @ w.t() for d, w in zip(parts(dY), W.double())])
    terms = torch.cat([d.abs() @ w.abs().t() for d, w in zip(parts(dY), W.double())])
    close(dX, want, sum_bound(terms, N) + rounding(want, dtype) * 1.01, "dX")
    work = torch.full((max(16, G.groot_grouped_product_backward_weights_workspace(n, E, K, N, dtype)),), 255, dtype=torch.uint8, device="cuda")
    dW, db = torch.full((E, K, N), float("nan"), device="cuda").to(dtype), torch.full((E, N), float("nan"), device="cuda").to(dtype)
    G.groot_grouped_product_backward_weights(X, dY, offsets, dW, db, work)
    rows = torch.tensor(sizes, device="cuda", dtype=torch.float64)
    want = torch.stack([x.t() @ d for x, d in zip(parts(X), parts(dY))])
    terms = torch.stack([x.abs().t() @ d.abs() for x, d in zip(parts(X), parts(dY))])
    close(dW, want, sum_bound(terms, rows[:, None, None]) + rounding(want, dtype) * 1.01, "dW")
    want = torch.stack([d.sum(0) for d in parts(dY)])
    terms = torch.stack([d.abs().sum(0) for d in parts(dY)])
    close(db, want, sum_bound(terms, rows[:, None]) + rounding(want, dtype) * 1.01, "db")


# around the borders of the pieces of 512 rows or more that a group's rows are cut into, in tiles of 64, 128 and 256, rows that begin
# on 16 bytes and that do not: (sizes of the groups, K, N, pad of the rows)
PIECES = [([n], 64, 64, 0) for n in (1, 511, 512, 513, 1023, 1024, 1025)] + [
    ([512 * 5 - 1, 512 * 3, 512 * 2 + 1, 0, 1, 512], 64, 48, 0), ([1537, 511, 2048], 60, 33, 1), ([20000], 64, 96, 0), ([9000], 20, 12, 0),
    ([9001], 20, 12, 1), ([8192, 8193], 72, 136, 0), ([2049, 0, 4095, 1], 200, 300, 0), ([2047, 0, 4097, 1], 200, 300, 1), ([33000, 511], 200, 200, 0),
    ([5000] + [60] * 15, 1024, 1024, 0), ([60] * 15 + [6145], 1024, 1024, 0), ([8192], 4096, 4096, 0), ([70000, 3, 66001], 32, 32, 0),
    ([600000], 16, 32, 0), ([524289, 524288], 48, 5, 0)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(PIECES)))
def test_weight_gradients_lose_no_row(kind, case):
    """Small integers: every partial sum is a whole number below 2^24, so that dW and dbias are exact, whatever the order, and a row
    that is left out or taken twice shows."""
    dtype, (sizes, K, N, pad) = TYPES[kind], PIECES[case]
    n, E = sum(sizes), len(sizes)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(500 + case)
    X = torch.randint(1, 3, (n, K + pad), generator=gen, device="cuda").to(dtype)[:, pad // 2:pad // 2 + K]
    dY = torch.randint(-2, 3, (n, N + pad), generator=gen, device="cuda").to(dtype)[:, pad // 2:pad // 2 + N]
    dY[:, 0] = 1                                             # a column of ones: the sums of X's columns, and the number of rows
    work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(n, E, K, N, dtype)), dtype=torch.uint8, device="cuda")
    want = torch.stack([x.double().t() @ d.double() for x, d in zip(X.split(sizes), dY.split(sizes))])
    want_db = torch.stack([d.double().sum(0) for d in dY.split(sizes)])
    for offsets in [offsets_of(sizes)] + [None] * (E == 1):
        for junk in (0, 255):
            dW, db = torch.full((E, K, N), float("nan"), device="cuda"), torch.full((E, N), float("nan"), device="cuda")
            work.fill_(junk)
            G.groot_grouped_product_backward_weights(X, dY, offsets, dW, db, work)
            assert torch.equal(dW.double(), want), int((dW.double() != want).sum())
            assert torch.equal(db.double(), want_db), int((db.double() != want_db).sum())


@pytest.mark.parametrize("case", range(len(LARGE)))
def test_quantized_product_large_sizes(case):
    sizes, K, N = LARGE[case]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(400 + case)
    n, E = sum(sizes), len(sizes)
    Q = torch.randint(-127, 128, (n, K), generator=gen, device="cuda", dtype=torch.int8)
    W = torch.randint(-127, 128, (E, N, K), generator=gen, device="cuda", dtype=torch.int8)
    qs, ws = torch.rand(n, generator=gen, device="cuda") * 0.01, torch.rand((E, N), generator=gen, device="cuda") * 0.01
    Y = out_matrix(n, N, torch.float32)
    G.groot_quantized_product(Q, qs, W, ws, offsets_of(sizes) if E > 1 else None, None, False, Y)
    dots = torch.cat([q @ w.t() for q, w in zip(Q.double().split(sizes), W.double())])
    want = dots * qs.double()[:, None] * ws.double()[group_of(sizes)]
    close(Y, want, 4 * 2.0 ** -24 * want.abs(), "Y")


def test_few_rows_of_many_groups_and_columns():
    """more workgroups than a launch holds, were few rows taken by themselves; small integers, whose sums are exact"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)

    def small(*shape, dtype):
        return torch.randint(-2, 3, shape, generator=gen, device="cuda", dtype=torch.int8).to(dtype)
    n, E, K, N = 16384, 1024, 65536, 16
    dY, W, offsets = small(n, N, dtype=torch.bfloat16), small(E, K, N, dtype=torch.bfloat16), offsets_of([16] * E)
    dX = out_matrix(n, K, torch.bfloat16)
    G.groot_grouped_product_backward_data(dY, W, offsets, dX)
    for g in range(0, E, 93):
        assert torch.equal(dX[16 * g:16 * g + 16].float(), dY[16 * g:16 * g + 16].float() @ W[g].float().t().contiguous()), g
    assert torch.isfinite(dX).all()
    del dY, W, dX
    n, E, K, N = 32768, 2048, 16, 32768
    Q, W, ones, scales = small(n, K, dtype=torch.int8), small(E, N, K, dtype=torch.int8), torch.ones(n, device="cuda"), torch.ones((E, N), device="cuda")
    Y = out_matrix(n, N, torch.bfloat16)
    G.groot_quantized_product(Q, ones, W, scales, offsets_of([16] * E), None, False, Y)
    for g in range(0, E, 178):
        assert torch.equal(Y[16 * g:16 * g + 16].float(), Q[16 * g:16 * g + 16].float() @ W[g].float().t().contiguous()), g
    assert torch.isfinite(Y).all()
    del Q, W, Y, scales
    E, K, N = 2048, 8, 65536
    X, W, scales = small(1, K, dtype=torch.float32), small(E, N, K, dtype=torch.int8), torch.ones((E, N), device="cuda")
    X[0, 0] = 2.0
    Y, work = out_matrix(1, N, torch.float32), torch.empty(G.groot_quantized_linear_workspace(1, K), dtype=torch.uint8, device="cuda")
    G.groot_quantized_linear(X, W, scales, offsets_of([0] * 1500 + [1] + [0] * (E - 1501)), None, False, Y, work)
    q, top = quantized(X)
    want = (q.double() @ W[1500].double().t()) * top.double()[:, None]
    close(Y, want, 4 * 2.0 ** -24 * want.abs(), "Y")


@pytest.mark.parametrize("kind", TYPES)
def test_no_rows_at_all(kind):
    dtype = TYPES[kind]
    X, dY, W = torch.empty((0, 40), dtype=dtype, device="cuda"), torch.empty((0, 24), dtype=dtype, device="cuda"), torch.ones((3, 40, 24), dtype=dtype, device="cuda")
    offsets = torch.zeros(4, dtype=torch.int64, device="cuda")
    G.groot_grouped_product(X, W, offsets, None, False, dY)
    G.groot_grouped_product_backward_data(dY, W, offsets, X)
    for many in (offsets, None):
        E = 3 if many is not None else 1
        dW, db = torch.full((E, 40, 24), 7.0, device="cuda").to(dtype), torch.full((E, 24), 7.0, device="cuda").to(dtype)
        G.groot_grouped_product_backward_weights(X, dY, many, dW, db, None)
        assert not dW.any() and not db.any()
    Q, W8 = torch.empty((0, 40), dtype=torch.int8, device="cuda"), torch.ones((3, 24, 40), dtype=torch.int8, device="cuda")
    s, ws = torch.empty(0, device="cuda"), torch.ones((3, 24), device="cuda")
    G.groot_quantize_rows(X, Q, s)
    G.groot_quantized_product(Q, s, W8, ws, offsets, None, False, dY)
    G.groot_quantized_linear(X, W8, ws, offsets, None, False, dY, torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_rows_far_apart():
    """element offsets beyond 2^32"""
    stride, n, K, N = (1 << 27) + 8, 40, 64, 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    small = matrix(gen, n, K, torch.bfloat16)
    far = torch.empty((n - 1) * stride + K, dtype=torch.bfloat16, device="cuda").as_strided((n, K), (stride, 1))
    far.copy_(small)
    W = matrix(gen, K, N, torch.bfloat16)[None].contiguous()
    Y, Z = out_matrix(n, N, torch.bfloat16), out_matrix(n, N, torch.bfloat16)
    G.groot_grouped_product(small, W, None, None, False, Y)
    G.groot_grouped_product(far, W, None, None, False, Z)
    assert torch.equal(Y, Z)
    dW, dV = (torch.empty((1, K, N), device="cuda") for _ in range(2))
    work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(n, 1, K, N, torch.bfloat16)), dtype=torch.uint8, device="cuda")
    G.groot_grouped_product_backward_weights(small, Y, None, dW, None, work)
    G.groot_grouped_product_backward_weights(far, Y, None, dV, None, work)
    assert torch.equal(dW, dV)
    del far
    q = torch.randint(-127, 128, (n, K), generator=gen, device="cuda", dtype=torch.int8)
    far = torch.empty((n - 1) * stride + K, dtype=torch.int8, device="cuda").as_strided((n, K), (stride, 1))
    far.copy_(q)
    w = torch.randint(-127, 128, (1, N, K), generator=gen, device="cuda", dtype=torch.int8)
    s, ws = torch.rand(n, generator=gen, device="cuda"), torch.rand((1, N), generator=gen, device="cuda")
    A, B = out_matrix(n, N, torch.float32), out_matrix(n, N, torch.float32)
    G.groot_quantized_product(q, s, w, ws, None, None, False, A)
    G.groot_quantized_product(far, s, w, ws, None, None, False, B)
    assert torch.equal(A, B)


# ---------------------------------------------------------------------------------------------------------------
# 8-bit products
# ---------------------------------------------------------------------------------------------------------------
def quantized(X):
    """fp32, operation by operation as the call states them"""
    x = X.float()
    top = x.abs().amax(1) / 127
    q = torch.where(top[:, None] > 0, torch.round(x / top[:, None]), torch.zeros_like(x))
    return q.to(torch.int8), top


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n, K, pad", [(1, 1, 0), (1, 4096, 0), (5, 63, 1), (70, 64, 0), (33, 1000, 8), (300, 257, 0), (9, 8200, 0)])
def test_quantize_rows(kind, n, K, pad):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + K)
    X = matrix(gen, n, K, TYPES[kind], pad)
    X[n // 2] = 0
    Q = torch.full((n, K + pad), 99, dtype=torch.int8, device="cuda")[:, :K]
    scale = torch.empty(n, device="cuda")
    G.groot_quantize_rows(X, Q, scale)
    q, top = quantized(X)
    assert torch.equal(scale, top) and torch.equal(Q, q)
    X[0, K - 1], X[n - 1, 0] = float("nan"), float("inf")
    G.groot_quantize_rows(X, Q, scale)
    bad = {0, n - 1}
    keep = [r for r in range(n) if r not in bad]
    assert torch.equal(Q[keep], q[keep]) and torch.equal(scale[keep], top[keep])
    assert all(torch.isnan(scale[r]) and not Q[r].any() for r in bad)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_quantized_product(kind, case):
    dtype, (sizes, K, N, pad) = TYPES[kind], SHAPES[case]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(200 + case)
    n, E = sum(sizes), len(sizes)
    Q = torch.randint(-128, 128, (max(n, 1), K + pad), generator=gen, device="cuda", dtype=torch.int8)[:n, pad // 2:pad // 2 + K]
    W = torch.randint(-128, 128, (E, N, K), generator=gen, device="cuda", dtype=torch.int8)
    qs, ws = torch.rand(n, generator=gen, device="cuda") * 0.01, torch.rand((E, N), generator=gen, device="cuda") * 0.01
    b = torch.randn((E, N), generator=gen, device="cuda")
    offsets = offsets_of(sizes)
    of = group_of(sizes)
    for relu in (False, True):
        Y = out_matrix(n, N, dtype, pad)
        G.groot_quantized_product(Q, qs, W, ws, offsets, None if relu else b, relu, Y)
        dots = torch.cat([q @ w.t() for q, w in zip(Q.double().split(sizes), W.double())])
        want = dots * qs.double()[:, None] * ws.double()[of]
        bound = 4 * 2.0 ** -24 * want.abs()
        if not relu:
            bound = bound + 2.0 ** -24 * (want + b.double()[of]).abs()
            want = want + b.double()[of]
        else:
            want = want.clamp(min=0)
        close(Y, want, bound + rounding(want, dtype) * 1.01, "Y")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("K, N", [(64, 64), (200, 256), (77, 31), (1024, 640)])
def test_quantized_rows_are_the_same_in_every_batch(kind, K, N):
    """bit for bit what the call states: the sum in fp32, times the row's scale, times the column's, plus the bias, one rounding each
    and one to the output's type; so it does not matter how many rows are served together"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(K + N)
    Q = torch.randint(-127, 128, (5000, K), generator=gen, device="cuda", dtype=torch.int8)
    W = torch.randint(-127, 128, (1, N, K), generator=gen, device="cuda", dtype=torch.int8)
    qs, ws = torch.rand(5000, generator=gen, device="cuda"), torch.rand((1, N), generator=gen, device="cuda")
    b = torch.randn((1, N), generator=gen, device="cuda") * 1e4
    dots = (Q.double() @ W[0].double().t()).cpu().float()
    want = (dots * qs.cpu()[:, None] * ws.cpu() + b.cpu()).to(TYPES[kind])
    for n in (1, 4, 16, 17, 48, 300, 5000):
        Y = out_matrix(n, N, TYPES[kind])
        G.groot_quantized_product(Q[:n], qs[:n], W, ws, None, b, False, Y)
        assert torch.equal(Y.cpu(), want[:n]), (n, int((Y.cpu() != want[:n]).sum()))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("sizes, K, N", [([1], 4096, 1024), ([1], 100, 37), ([4], 513, 200), ([16], 1024, 512), ([17], 768, 260), ([48], 2048, 520),
                                         ([1, 0, 2, 1], 640, 96), ([130, 200], 256, 192), ([600], 1030, 390)])
def test_quantized_linear(kind, sizes, K, N):
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(K + N)
    n, E = sum(sizes), len(sizes)
    X = matrix(gen, n, K, dtype, 8)
    W = torch.randint(-127, 128, (E, N, K), generator=gen, device="cuda", dtype=torch.int8)
    ws, b = torch.rand((E, N), generator=gen, device="cuda") * 0.01, torch.randn((E, N), generator=gen, device="cuda")
    Y = out_matrix(n, N, dtype, 2)
    work = torch.empty(G.groot_quantized_linear_workspace(n, K), dtype=torch.uint8, device="cuda")
    G.groot_quantized_linear(X, W, ws, offsets_of(sizes) if E > 1 else None, b, False, Y, work)
    q, top = quantized(X)
    of = group_of(sizes)
    dots = torch.cat([x @ w.t() for x, w in zip(q.double().split(sizes), W.double())])
    want = dots * top.double()[:, None] * ws.double()[of]
    bound = 4 * 2.0 ** -24 * want.abs()
    want = want + b.double()[of]
    close(Y, want, bound + 2.0 ** -24 * want.abs() + rounding(want, dtype) * 1.01, "Y")
    Z = out_matrix(n, N, dtype)
    G.groot_quantized_product(q, top, W, ws, offsets_of(sizes) if E > 1 else None, b, False, Z)
    assert torch.equal(Y, Z), "the two ways differ"
    X[0, 0] = float("nan")
    G.groot_quantized_linear(X, W, ws, offsets_of(sizes) if E > 1 else None, b, False, Y, work)
    assert torch.isnan(Y[0]).all() and torch.equal(Y[1:], Z[1:])


# ---------------------------------------------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------------------------------------------
LR, B1, B2, EPS, WD = 3e-3, 0.9, 0.95, 1e-8, 0.1


def mixed(h):
    h = h & 0xFFFFFFFF
    h ^= h >> 16
    h = (h * 0x85EBCA6B) & 0xFFFFFFFF
    h ^= h >> 13
    h = (h * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def randoms(i, n, step, seed):
    key = mixed(mixed(mixed(i + 0x9E3779B9) ^ step) ^ seed)
    h = mixed(torch.arange(n, device="cuda") ^ key)
    return (h & 0xFFFF).double() / 65536, (h >> 16).double() / 65536


def on_grid(x, u):
    _, e = torch.frexp(x)
    step = torch.tensor([2.0 ** (k - 9) for k in range(16)], dtype=torch.float64, device="cuda")[torch.clamp(e, -5, 10).long() + 5]
    return torch.clamp(torch.floor(x.abs() / step + u) * step, max=448.0)


def adamw_case(sizes, param, grad, bits, master, seed, shift=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def flat(n, dtype, scale):
        whole = torch.zeros(n + 16, dtype=dtype, device="cuda")
        t = whole[shift:shift + n]
        t.copy_(torch.randn(n, generator=gen, device="cuda") * scale)
        return t
    s = dict(p=[flat(n, param, 0.1) for n in sizes], g=[flat(n, grad, 0.01) for n in sizes], master=None)
    if master:
        s["master"] = [flat(n, torch.float32, 0.1) for n in sizes]
    if bits == 32:
        s["m"], s["v"] = [flat(n, torch.float32, 0.005) for n in sizes], [flat(n, torch.float32, 0.01).square_() for n in sizes]
        return s
    for k in ("m", "v"):
        s[k + "_scale"] = [torch.rand(-(-n // 256), generator=gen, device="cuda") * 1e-4 for n in sizes]
        codes = [torch.randint(0, 0x7E if k == "v" else 256, (n + 16,), generator=gen, device="cuda") for n in sizes]
        s[k] = [torch.where((c & 0x7F) == 0x7F, 5, c).to(torch.uint8).view(torch.float8_e4m3fn)[shift:shift + n] for c, n in zip(codes, sizes)]
    return s


def adamw_run(s, step, seed=0, grad_scale=None):
    more = {k: s[k] for k in ("m_scale", "v_scale") if k in s}
    G.groot_adamw_step(G.groot_adamw_tensors(s["p"], s["g"], s["m"], s["v"], master=s["master"], **more), step, LR, B1, B2, EPS, WD,
                       grad_scale=grad_scale, seed=seed)


def adamw_check(s, old, step, seed=0, gs=1.0):
    """m and v: three roundings and a rounded factor for each term, of the terms' magnitudes.  w: the step's own relative error is
    that of m's terms, of the root (half of v's, and one), of a product, a sum, a division, a product and two factors: below
    16 x 2^-24; w itself is rounded with the factor, the product and the sum."""
    u = 2.0 ** -24
    for i in range(len(s["p"])):
        n = s["p"][i].numel()
        if n == 0:
            continue
        held = lambda k: old[k][i].double() * old[k + "_scale"][i].double().repeat_interleave(256)[:n] if "m_scale" in s else old[k][i].double()  # noqa: E731
        m0, v0, g = held("m"), held("v"), old["g"][i].double() * gs
        more = 2 * u if "m_scale" in s else 0.0                        # code * scale is rounded, the root once more when squared
        v0 = v0 * v0 if "m_scale" in s else v0
        m, v = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g
        m_terms = B1 * m0.abs() + (1 - B1) * g.abs()
        m_off, v_off = (4 * u + more) * m_terms, (6 * u + 3 * more) * v
        w0 = (old["p"][i] if s["master"] is None else old["master"][i]).double()
        denom = (v / (1 - B2 ** step)).sqrt() + EPS
        w = w0 * (1 - LR * WD) - LR / (1 - B1 ** step) * m / denom
        w_off = 4 * u * w0.abs() + (16 * u + 6 * more) * LR / (1 - B1 ** step) * m_terms / denom + u * w.abs()
        if s["master"] is not None:
            close(s["master"][i], w, w_off, f"master[{i}]")
            assert torch.equal(s["p"][i], s["master"][i].to(s["p"][i].dtype))
        else:
            close(s["p"][i], w, w_off + rounding(w, s["p"][i].dtype) * 1.01, f"p[{i}]")
        if "m_scale" not in s:
            close(s["m"][i], m, m_off + 1e-45, f"m[{i}]")
            close(s["v"][i], v, v_off + 1e-45, f"v[{i}]")
            continue
        um, uv = randoms(i, n, step, seed)
        for k, x, off, r in (("m", m, m_off, um), ("v", v.sqrt(), v.sqrt() * (4 * u + 3 * more), uv)):
            pad = -n % 256
            blocks = torch.nn.functional.pad(x.abs(), (0, pad)).reshape(-1, 256)
            top = blocks.amax(1)
            slack = torch.nn.functional.pad(off, (0, pad)).reshape(-1, 256).amax(1)
            close(s[k + "_scale"][i], top / 448, slack / 448 + 2 * u * top / 448, f"{k}_scale[{i}]")
            scale = s[k + "_scale"][i].double().repeat_interleave(256)[:n]
            over, eps = x.abs() / scale, off / scale + 2 * u * x.abs() / scale
            low, high = on_grid((over - eps).clamp(min=0), r - 2.0 ** -19), on_grid(over + eps, r + 2.0 ** -19)
            if k == "v":
                low, high = low.clamp(min=2.0 ** -9), high.clamp(min=2.0 ** -9)
            got = s[k][i].double()
            bad = (got.abs() < low) | (got.abs() > high) | ((got != 0) & (torch.sign(got) != torch.sign(x)) & (x.abs() > off))
            assert int(bad.sum()) == 0, f"{k}[{i}]: {[(j, float(got[j]), float(over[j]), float(r[j])) for j in bad.nonzero()[:4, 0].tolist()]}"


def clone(s):
    return {k: None if x is None else [t.clone() for t in x] for k, x in s.items()}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param, grad, master", [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", True), ("bf16", "f32", False),
                                                 ("f16", "f16", True), ("f16", "f16", False), ("f32", "f16", True)])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw(bits, param, grad, master, shift):
    sizes = [1, 3, 255, 256, 257, 0, 1024, 2048, 2049, 70000, 5] + [64] * 60
    s = adamw_case(sizes, TYPES[param], TYPES[grad], bits, master, 11, shift)
    for step in (1, 2, 1000):
        old = clone(s)
        adamw_run(s, step, seed=77)
        adamw_check(s, old, step, seed=77)


def adamw_fp32(s, step, lr, b1, b2, eps, wd):
    """the new weights, every operation in fp32 by itself, on the CPU, in the order that the call states"""
    cut = lambda x: torch.tensor(np.float32(x))  # noqa: E731
    out = []
    for i, g in enumerate(s["g"]):
        g, n = g.cpu().float(), g.numel()
        m, v = (s[k][i].cpu().float() for k in ("m", "v"))
        if "m_scale" in s:
            m, v = (x * s[k][i].cpu().repeat_interleave(256)[:n] for x, k in ((m, "m_scale"), (v, "v_scale")))
            v = v * v
        m = m * cut(b1) + g * cut(1 - b1)
        v = v * cut(b2) + (g * g) * cut(1 - b2)
        root = v.double().sqrt().float()                     # rounded once (the CPU's own root of fp32 tensors is off by a place here and there)
        denom = root * cut(1 / math.sqrt(1 - b2 ** step)) + cut(eps)
        w = (s["p"] if s["master"] is None else s["master"])[i].cpu().float()
        out.append(w * cut(1 - lr * wd) - cut(lr / (1 - b1 ** step)) * (m / denom))
    return out


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param, grad, master", [("f32", "f32", False), ("bf16", "bf16", True)])
@pytest.mark.parametrize("weights", [0.0, 1.0])
def test_adamw_rounds_every_operation_by_itself(bits, param, grad, master, weights):
    """bit for bit: in 8 bits as in 32, and where values lie outside the range of the short divisions"""
    for eps, spread in ((1e-8, 1.0), (1e-39, 1.0), (1e-8, 1e-18), (1e-3, 1e12)):
        s = adamw_case([400000, 1001], TYPES[param], TYPES[grad], bits, master, 21)
        for k in ("p", "master"):
            for t in s[k] or []:
                t.mul_(weights)
        for t in s["g"]:
            t.mul_(spread)
        if bits == 8:
            for t in s["m_scale"] + s["v_scale"]:
                t.mul_(spread)
        for k, power in (("m", 1), ("v", 2)):
            if bits == 32:
                for t in s[k]:
                    t.mul_(spread ** power)
        s["g"][1][:600] = 0                                  # two blocks that hold nothing, and one in part
        s["m"][1][:600] = torch.zeros(600, device="cuda").to(s["m"][1].dtype)
        s["v"][1][:600] = torch.zeros(600, device="cuda").to(s["v"][1].dtype)
        want = adamw_fp32(s, 3, LR, B1, B2, eps, WD)
        more = {k: s[k] for k in ("m_scale", "v_scale") if k in s}
        G.groot_adamw_step(G.groot_adamw_tensors(s["p"], s["g"], s["m"], s["v"], master=s["master"], **more), 3, LR, B1, B2, eps, WD, seed=4)
        for i, w in enumerate(want):
            got = (s["p"] if s["master"] is None else s["master"])[i].cpu()
            assert torch.isfinite(got).all()
            assert torch.equal(got, w), (eps, spread, i, int((got != w).sum()), w.numel())


def test_adamw_tensors_that_move():
    def make():
        return adamw_case([300, 20, 5000], torch.float32, torch.float32, 32, False, 5)

    def tensors_of(s):
        return G.groot_adamw_tensors(s["p"], s["g"], s["m"], s["v"])
    for k in ("p", "g", "m", "v"):
        s = make()
        tensors = tensors_of(s)
        for step in range(1, 30):
            G.groot_adamw_step(tensors, step, LR)
        s[k][1].data = s[k][1].clone()
        with pytest.raises(RuntimeError, match="moved"):
            for step in range(30, 60):
                G.groot_adamw_step(tensors, step, LR)
        old = clone(s)
        G.groot_adamw_step(tensors_of(s), 7, LR, B1, B2, EPS, WD)
        adamw_check(s, old, 7)
    s, t = make(), make()
    tensors = tensors_of(s)
    s["g"] = t["g"] = [g * 0.5 for g in s["g"]]              # as autograd makes them anew
    tensors.set_grads(s["g"])
    for step in range(1, 30):
        G.groot_adamw_step(tensors, step, LR)
        G.groot_adamw_step(tensors_of(t), step, LR)
    assert all(torch.equal(a, b) for k in ("p", "m", "v") for a, b in zip(s[k], t[k]))


def test_adamw_gradient_scale_and_repeats():
    for bits in (32, 8):
        s = adamw_case([1000, 300], torch.float32, torch.float32, bits, False, 3)
        old, t = clone(s), clone(s)
        adamw_run(s, 5, seed=1, grad_scale=torch.tensor([0.25], device="cuda"))
        adamw_check(s, old, 5, seed=1, gs=0.25)
        adamw_run(t, 5, seed=1, grad_scale=torch.tensor(0.25, device="cuda"))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for k in ("p", "m", "v") for a, b in zip(s[k], t[k]))


def test_adamw_of_a_tensor_beyond_32_bits(monkeypatch):
    """the values, codes, scales and random numbers about the place 2^32 of one tensor, and at its ends"""
    n, step, seed = (1 << 32) + 1300, 6, 9
    zeros = lambda k, dtype: torch.zeros(k, dtype=dtype, device="cuda")  # noqa: E731
    bf16, codes = torch.bfloat16, torch.float8_e4m3fn
    s = dict(p=[zeros(n, bf16)], g=[zeros(n, bf16)], m=[zeros(n, torch.uint8).view(codes)], v=[zeros(n, torch.uint8).view(codes)],
             m_scale=[zeros(-(-n // 256), torch.float32)], v_scale=[zeros(-(-n // 256), torch.float32)], master=None)
    places = [(0, 1024), ((1 << 31) - 512, (1 << 31) + 512), ((1 << 32) - 1024, n)]        # whole blocks, but the last
    part = lambda x, k, a, b: x[k][0][a // 256:-(-b // 256)] if "scale" in k else x[k][0][a:b]  # noqa: E731
    olds = []
    for seed_of, (a, b) in enumerate(places):
        here = adamw_case([b - a], bf16, bf16, 8, False, 40 + seed_of)
        for k in s:
            if s[k] is not None:
                part(s, k, a, b).view(torch.uint8).copy_(here[k][0].view(torch.uint8))
        olds.append(here)
    G.groot_adamw_step(G.groot_adamw_tensors(s["p"], s["g"], s["m"], s["v"], m_scale=s["m_scale"], v_scale=s["v_scale"]), step, LR, B1, B2, EPS, WD, seed=seed)
    for (a, b), old in zip(places, olds):
        def randoms_here(i, count, step, seed):
            at = torch.arange(a, b, device="cuda")
            key = mixed(mixed(mixed(i + 0x9E3779B9) ^ step) ^ seed)
            h = mixed((at & 0xFFFFFFFF) ^ ((key + (at >> 32) * 0x9E3779B9) & 0xFFFFFFFF))
            return (h & 0xFFFF).double() / 65536, (h >> 16).double() / 65536
        monkeypatch.setattr(sys.modules[__name__], "randoms", randoms_here)
        adamw_check({k: None if s[k] is None else [part(s, k, a, b)] for k in s}, old, step, seed)
    for a, b in ((1024, 1 << 20), ((1 << 31) + 512, (1 << 31) + (1 << 20)), ((1 << 32) - (1 << 20), (1 << 32) - 1024)):
        assert not any(s[k][0][a:b].view(torch.uint8).any() for k in ("p", "m", "v"))       # what lies between stayed


def test_adamw_values_that_are_not_finite():
    for bits in (32, 8):
        s, t = (adamw_case([600], torch.float32, torch.float32, bits, False, 3) for _ in range(2))
        s["g"][0][[7, 300]] = torch.tensor([float("nan"), float("inf")], device="cuda")
        t["g"][0][[7, 300]] = 0
        before = clone(s)
        adamw_run(s, 2)
        adamw_run(t, 2)
        keep = torch.ones(600, dtype=torch.bool, device="cuda")
        keep[[7, 300]] = False
        assert torch.equal(s["p"][0][keep], t["p"][0][keep])
        assert not torch.isfinite(s["p"][0][[7, 300]]).any()
        if bits == 8:
            assert torch.isnan(s["m"][0][[7, 300]].float()).all() and torch.isnan(s["v"][0][[7, 300]].float()).all()
            assert torch.isfinite(s["m"][0].float()[keep]).all() and torch.isfinite(s["m_scale"][0]).all()
        del before
    s = adamw_case([512], torch.float32, torch.float32, 8, False, 3)
    for x in (s["g"], s["m_scale"], s["v_scale"]):
        x[0].zero_()
    w = s["p"][0].clone()
    adamw_run(s, 1)                                       # nothing but weight decay
    close(s["p"][0], w.double() * (1 - LR * WD), 4 * 2.0 ** -24 * w.abs().double(), "p")
    assert not s["m"][0].view(torch.uint8).bitwise_and(0x7F).any() and not s["m_scale"][0].any()


def test_adamw_8_bits_follows_32():
    """A quadratic with its own curvature for every value: states in 8 bits reach the loss that 32 bits reach, within a factor of 1.5
    of what is left, where states rounded to nearest would stand still."""
    n, steps = 4096, 400
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    curve = torch.exp(torch.randn(n, generator=gen, device="cuda"))
    start = torch.randn(n, generator=gen, device="cuda")
    left = {}
    for bits in (32, 8):
        p = start.clone()
        zeros = lambda: torch.zeros(n, device="cuda")  # noqa: E731
        more, m, v = {}, zeros(), zeros()
        if bits == 8:
            m, v = m.to(torch.float8_e4m3fn), v.to(torch.float8_e4m3fn)
            more = dict(m_scale=[torch.zeros(16, device="cuda")], v_scale=[torch.zeros(16, device="cuda")])
        g = torch.empty(n, device="cuda")
        tensors = G.groot_adamw_tensors([p], [g], [m], [v], **more)
        for t in range(1, steps + 1):
            torch.mul(curve, p, out=g)
            G.groot_adamw_step(tensors, t, 1e-2 * (1 - t / (steps + 1)), 0.9, 0.999, 1e-8, 0.0, seed=5)
        left[bits] = float((curve * p * p).sum())
    whole = float((curve * start * start).sum())
    assert left[32] < 0.1 * whole
    assert left[8] < 1.5 * left[32] + 1e-3 * whole, left


# ---------------------------------------------------------------------------------------------------------------
# streams, graphs
# ---------------------------------------------------------------------------------------------------------------
def test_on_a_stream_of_its_own_and_replayed_from_a_graph():
    sizes, K, N = [100, 0, 260], 64, 96
    dtype = torch.bfloat16
    n, E, X, dY, W, b = case_tensors(dtype, sizes, K, N, 0, 8)
    offsets = offsets_of(sizes)
    Y, dX, dW, db = out_matrix(n, N, dtype), out_matrix(n, K, dtype), torch.empty((E, K, N), dtype=dtype, device="cuda"), torch.empty((E, N), dtype=dtype, device="cuda")
    work = torch.empty(max(16, G.groot_grouped_product_backward_weights_workspace(n, E, K, N, dtype)), dtype=torch.uint8, device="cuda")
    Wq = torch.randint(-127, 128, (E, N, K), device="cuda", dtype=torch.int8)
    ws = torch.rand((E, N), device="cuda") * 0.01
    Z, qwork = out_matrix(n, N, dtype), torch.empty(G.groot_quantized_linear_workspace(n, K), dtype=torch.uint8, device="cuda")
    m, v = torch.zeros((E, K, N), device="cuda"), torch.zeros((E, K, N), device="cuda")
    p = W.clone()
    tensors = G.groot_adamw_tensors([p], [dW], [m], [v])

    def step():
        G.groot_grouped_product(X, p, offsets, b, True, Y)
        G.groot_grouped_product_backward_data(dY, p, offsets, dX)
        G.groot_grouped_product_backward_weights(X, dY, offsets, dW, db, work)
        G.groot_quantized_linear(X, Wq, ws, offsets, None, False, Z, qwork)
        G.groot_adamw_step(tensors, 1, 1e-2)
    outs = (Y, dX, dW, db, Z, p, m, v)

    def begin():
        p.copy_(W), m.zero_(), v.zero_(), X.mul_(-1)
    wanted = []
    for _ in range(4):
        begin()
        step()
        wanted.append([t.clone() for t in outs])
    side = torch.cuda.Stream()
    begin()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(outs, wanted[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(1, 4):
        begin()
        for t in (Y, dX, dW, db, Z):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs, wanted[k])), k
        torch.randn(1000, device="cuda").sum().item()


FIRST_CALL_CAPTURED = """
import torch
import paper_2511_18297_amd as G
gen = torch.Generator(device="cuda")
gen.manual_seed(1)
cases = []
for dtype, n, K, N, pad in ((torch.float32, 4096, 64, 64, 0), (torch.float32, 4096, 128, 128, 0), (torch.bfloat16, 4096, 200, 100, 0), (torch.float16, 4096, 250, 120, 1)):
    X = torch.randint(-2, 3, (n, K + pad), generator=gen, device="cuda").to(dtype)[:, :K]
    W = torch.randint(-1, 2, (1, K, N), generator=gen, device="cuda").to(dtype)
    cases.append((X, W, torch.empty((n, N), dtype=dtype, device="cuda")))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for X, W, Y in cases:
        G.groot_grouped_product(X, W, None, None, False, Y)
for replay in range(3):
    for X, W, Y in cases:
        X.mul_(-1)
        Y.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    for X, W, Y in cases:
        want = X.double() @ W[0].double()
        assert (Y.double() - want).abs().max() <= 2.0 ** -8 * want.abs().max(), (replay, Y.dtype)
print("captured")
"""


def test_narrow_rows_whose_first_call_is_captured():
    """in a process that has not called them: nothing has to be asked of the runtime before"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALL_CAPTURED], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]
