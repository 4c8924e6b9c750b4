"""What the grouped products, the 8-bit products and the AdamW step refuse, before anything reaches a device."""
import ctypes

import pytest
import torch
from torch.multiprocessing.reductions import StorageWeakRef

from util import ensure_built

ensure_built()
import paper_2511_18297_amd as G  # noqa: E402

L = G.binding._lib
MB = 1 << 20


class Buffers:
    """Addresses that are never read: a few megabytes apart, 256-byte aligned."""

    def __init__(self):
        self.at = 1 << 30

    def __call__(self, mb=1):
        p = self.at
        self.at += mb * MB
        return p


def grouped(**change):
    b = Buffers()
    a = dict(dtype=1, X=b(), xs=64, W=b(), off=b(), bias=b(), relu=0, Y=b(), ys=32, n=100, E=3, K=64, N=32)
    a.update(change)
    return L.groot_grouped_product(a["dtype"], a["X"], a["xs"], a["W"], a["off"], a["bias"], a["relu"], a["Y"], a["ys"], a["n"], a["E"], a["K"], a["N"], None)


def data(**change):
    b = Buffers()
    a = dict(dtype=1, dY=b(), dys=32, W=b(), off=b(), dX=b(), dxs=64, n=100, E=3, K=64, N=32)
    a.update(change)
    return L.groot_grouped_product_backward_data(a["dtype"], a["dY"], a["dys"], a["W"], a["off"], a["dX"], a["dxs"], a["n"], a["E"], a["K"], a["N"], None)


def weights(**change):
    b = Buffers()
    a = dict(dtype=1, X=b(), xs=64, dY=b(), dys=32, off=b(), gd=0, dW=b(), db=b(), n=100, E=3, K=64, N=32, ws=b(512), wb=512 * MB)
    a.update(change)
    return L.groot_grouped_product_backward_weights(a["dtype"], a["X"], a["xs"], a["dY"], a["dys"], a["off"], a["gd"], a["dW"], a["db"], a["n"], a["E"],
                                                    a["K"], a["N"], a["ws"], a["wb"], None)


def quantize(**change):
    b = Buffers()
    a = dict(dtype=1, X=b(), xs=64, Q=b(), qs=64, s=b(), n=100, K=64)
    a.update(change)
    return L.groot_quantize_rows(a["dtype"], a["X"], a["xs"], a["Q"], a["qs"], a["s"], a["n"], a["K"], None)


def product(**change):
    b = Buffers()
    a = dict(Q=b(), qs=64, s=b(), W=b(), w=b(), off=b(), bias=b(), relu=0, dtype=1, Y=b(), ys=32, n=100, E=3, K=64, N=32)
    a.update(change)
    return L.groot_quantized_product(a["Q"], a["qs"], a["s"], a["W"], a["w"], a["off"], a["bias"], a["relu"], a["dtype"], a["Y"], a["ys"], a["n"], a["E"],
                                     a["K"], a["N"], None)


def linear(**change):
    b = Buffers()
    a = dict(dtype=1, X=b(), xs=64, W=b(), w=b(), off=b(), bias=b(), relu=0, Y=b(), ys=32, n=100, E=3, K=64, N=32, ws=b(), wb=MB)
    a.update(change)
    return L.groot_quantized_linear(a["dtype"], a["X"], a["xs"], a["W"], a["w"], a["off"], a["bias"], a["relu"], a["Y"], a["ys"], a["n"], a["E"], a["K"],
                                    a["N"], a["ws"], a["wb"], None)


SIZES = [dict(n=-1), dict(E=0), dict(E=70000), dict(K=0), dict(N=0), dict(K=65537, xs=70000, dxs=70000, qs=70000), dict(N=65537, ys=70000, dys=70000),
         dict(off=None), dict(off=(1 << 30) + 4)]
FIRST = 1 << 30                                            # where the first buffer lies


@pytest.mark.parametrize("call, more", [
    (grouped, [dict(dtype=3), dict(dtype=-1), dict(X=None), dict(W=None), dict(Y=None), dict(xs=63), dict(ys=31), dict(relu=2), dict(X=FIRST + 1),
               dict(bias=FIRST + 1), dict(Y=FIRST + 128), dict(xs=1 << 62), dict(n=1 << 41)]),
    (data, [dict(dtype=9), dict(dY=None), dict(W=None), dict(dX=None), dict(dys=31), dict(dxs=63), dict(dX=FIRST)]),
    (weights, [dict(dtype=7), dict(gd=2), dict(X=None), dict(dY=None), dict(dW=None), dict(xs=63), dict(dys=31), dict(dW=FIRST), dict(db=FIRST),
               dict(dW=FIRST + 2 * MB + 2)]),
    (product, [dict(dtype=4), dict(Q=None), dict(s=None), dict(W=None), dict(w=None), dict(Y=None), dict(qs=63), dict(ys=31), dict(relu=-1),
               dict(w=FIRST + 2), dict(Y=FIRST)]),
    (linear, [dict(dtype=4), dict(X=None), dict(W=None), dict(w=None), dict(Y=None), dict(ws=None), dict(wb=100), dict(ws=FIRST + 8), dict(ws=FIRST),
              dict(Y=FIRST)]),
])
def test_refused(call, more):
    for change in SIZES + more:
        assert call(**change) == G.GROOT_EINVAL, change
        assert G.groot_last_error().startswith("groot_"), change


def test_quantize_refused():
    for change in (dict(dtype=3), dict(X=None), dict(Q=None), dict(s=None), dict(xs=63), dict(qs=63), dict(K=0), dict(K=70000), dict(n=-3), dict(Q=FIRST + 64),
                   dict(s=FIRST + 64), dict(X=FIRST + 1)):
        assert quantize(**change) == G.GROOT_EINVAL, change


def test_too_many_tiles():
    assert grouped(n=1 << 34, N=65536, ys=65536, Y=1 << 52) == G.GROOT_ERANGE
    assert product(n=1 << 34, N=65536, ys=65536, Y=1 << 52) == G.GROOT_ERANGE
    assert weights(E=65536, K=65536, N=65536, xs=65536, dys=65536, n=0, dW=1 << 52, db=1 << 56, ws=1 << 58, wb=1 << 40) == G.GROOT_ERANGE


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls pass the checks, and their addresses are not memory")
def test_few_rows_of_many_groups_are_not_refused():
    """more workgroups than a launch holds where few rows would go by themselves; the tiles hold them"""
    assert data(n=16384, E=1024, K=65536, N=16, dys=16, dxs=65536, dX=1 << 44, W=1 << 45) != G.GROOT_ERANGE
    assert product(n=32768, E=2048, K=16, N=32768, qs=16, ys=32768, Y=1 << 44, W=1 << 45) != G.GROOT_ERANGE
    assert linear(n=1, E=2048, K=8, N=65536, xs=8, ys=65536, Y=1 << 44, W=1 << 45, w=1 << 46, bias=None) != G.GROOT_ERANGE


def test_nothing_to_do():
    assert grouped(n=0) == data(n=0) == product(n=0) == linear(n=0) == quantize(n=0) == G.GROOT_OK


def test_workspaces():
    b = ctypes.c_size_t(77)
    for args in ((5, 10, 1, 8, 8), (0, -1, 1, 8, 8), (0, 10, 0, 8, 8), (0, 10, 1, 0, 8), (0, 10, 1, 8, 65537)):
        assert L.groot_grouped_product_backward_weights_workspace(*args, ctypes.byref(b)) == G.GROOT_EINVAL and b.value == 77
    assert L.groot_grouped_product_backward_weights_workspace(0, 10, 1, 8, 8, None) == G.GROOT_EINVAL
    assert L.groot_quantized_linear_workspace(10, 0, ctypes.byref(b)) == G.GROOT_EINVAL and b.value == 77
    assert G.groot_quantized_linear_workspace(10, 64) == 10 * 68
    need = G.groot_grouped_product_backward_weights_workspace(1 << 20, 3, 64, 32, torch.float32)   # the sizes of weights()
    if need:
        assert weights(dtype=0, n=1 << 20, wb=need - 1, X=1 << 40, dY=1 << 42) == G.GROOT_EINVAL


def adamw(n=1, pd=0, gd=0, bits=32, step=1, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, gs=None, tensors=None, count=None):
    array = (G.binding._AdamwTensor * max(n, 1))()
    for i in range(n):
        b = Buffers()
        for name in ("param", "grad", "m", "v", "m_scale", "v_scale"):
            setattr(array[i], name, b())
        array[i].n = 10
        for name, value in (tensors or {}).items():
            setattr(array[i], name, value)
    if n == 2 and tensors and "master" in tensors:
        array[1].master = None
    return L.groot_adamw_step(array, n if count is None else count, pd, gd, bits, step, lr, b1, b2, eps, wd, gs, 0, None)


def test_adamw_refused():
    inf, nan = float("inf"), float("nan")
    for change in (dict(pd=3), dict(gd=-1), dict(bits=16), dict(step=0), dict(step=-4), dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(b1=1.0), dict(b1=-0.1),
                   dict(b1=nan), dict(b2=1.0), dict(eps=0.0), dict(eps=nan), dict(eps=-1e-8), dict(wd=-0.1), dict(wd=nan), dict(gs=(1 << 30) + 2),
                   dict(count=-1), dict(tensors=dict(param=None)), dict(tensors=dict(grad=None)), dict(tensors=dict(m=None)), dict(tensors=dict(v=None)),
                   dict(tensors=dict(n=-1)), dict(bits=8, tensors=dict(m_scale=None)), dict(bits=8, tensors=dict(v_scale=None)),
                   dict(tensors=dict(param=(1 << 30) + 2)), dict(tensors=dict(m=(1 << 30) + 2)), dict(n=2, tensors=dict(master=1 << 40))):
        assert adamw(**change) == G.GROOT_EINVAL, change
    assert adamw(tensors=dict(n=1 << 40)) == G.GROOT_ERANGE
    assert adamw(n=0) == adamw(tensors=dict(n=0, param=None)) == G.GROOT_OK
    assert L.groot_adamw_step(None, 2, 0, 0, 32, 1, 1e-3, 0.9, 0.99, 1e-8, 0.0, None, 0, None) == G.GROOT_EINVAL


def test_adamw_refuses_factors_that_fp32_cannot_hold():
    """the kernel computes in fp32: an eps that is 0 there divides 0 by 0, a step of infinity multiplies 0 by it"""
    for change in (dict(eps=1e-60), dict(eps=1e-320), dict(eps=7e-46), dict(eps=1e39), dict(lr=1e300), dict(lr=4e38), dict(lr=1e37, b1=0.99),
                   dict(lr=1e20, wd=1e300), dict(lr=1e200, wd=1e200)):
        assert adamw(n=0, **change) == G.GROOT_EINVAL, change
        assert adamw(n=0, bits=8, **change) == G.GROOT_EINVAL, change
    for change in (dict(eps=1e-39), dict(eps=1.5e-45), dict(eps=3e38), dict(lr=1e37), dict(lr=0.0, wd=0.0), dict(lr=1e37, wd=10.0)):
        assert adamw(n=0, **change) == G.GROOT_OK, change


def test_binding_refuses_what_the_library_cannot_see():
    x, w, y = torch.zeros(4, 8), torch.zeros(1, 8, 8), torch.zeros(4, 8)
    with pytest.raises(TypeError):
        G.groot_grouped_product(x, w, None, None, False, y)          # not on the device
    with pytest.raises(TypeError):
        G.groot_grouped_product(x.double(), w, None, None, False, y)
    with pytest.raises(TypeError):
        G.groot_quantize_rows(x, y.to(torch.int8), torch.zeros(4))
    with pytest.raises(TypeError):
        G.groot_grouped_product_backward_weights_workspace(1, 1, 8, 8, torch.float64)
    with pytest.raises(ValueError):
        G.groot_adamw_tensors([x], [], [x], [x])
    with pytest.raises(ValueError):
        G.groot_adamw_tensors([x], [x], [x], [x], m_scale=[x])
    with pytest.raises(TypeError):
        G.groot_adamw_tensors([x], [x], [x], [x])


class OnDevice(torch.Tensor):
    """a tensor in host memory that calls itself one on the device: for checks that end before anything reads it"""
    is_cuda = True


def on_device(*shape, dtype=torch.float32):
    return torch.Tensor._make_subclass(OnDevice, torch.zeros(shape, dtype=dtype))


def test_refused_gradients_leave_the_descriptors_as_they_were():
    params, grads, m, v = ([on_device(300), on_device(20)] for _ in range(4))
    t = G.groot_adamw_tensors(params, grads, m, v)
    before = t.array.copy()
    bf16 = torch.bfloat16
    for bad, error in (([on_device(300, dtype=bf16), on_device(21, dtype=bf16)], ValueError), ([on_device(300, dtype=bf16), on_device(20)], TypeError),
                       ([on_device(300, dtype=bf16), torch.zeros(20, dtype=bf16)], TypeError), ([on_device(300, dtype=bf16)], ValueError)):
        with pytest.raises(error):
            t.set_grads(bad)
        assert t.grad_dtype == G.GROOT_F32 and (t.array == before).all()
    good = [on_device(300, dtype=bf16), on_device(20, dtype=bf16)]
    t.set_grads(good)
    assert t.grad_dtype == G.GROOT_BF16 and t.array[:, 1].tolist() == [g.data_ptr() for g in good]
    assert (t.array[:, [0, 2, 3, 4, 5, 6, 7]] == before[:, [0, 2, 3, 4, 5, 6, 7]]).all()


def test_descriptors_keep_the_memory_that_they_point_to():
    lists = {k: [on_device(300), on_device(300)] for k in ("params", "grads", "m", "v", "master")}
    t = G.groot_adamw_tensors(**lists)
    storages = [StorageWeakRef(x.untyped_storage()) for tensors in lists.values() for x in tensors]
    addresses = t.array.copy()
    for tensors in lists.values():
        for x in tensors:
            x.data = torch.zeros(7)                          # as Module.to does with its parameters
    assert not any(s.expired() for s in storages) and (t.array == addresses).all()
    del t
    assert all(s.expired() for s in storages)


def test_arrays_that_overlap():
    def make(**change):
        lists = dict(params=[on_device(300), on_device(20)], grads=[on_device(300), on_device(20)], m=[on_device(300), on_device(20)],
                     v=[on_device(300), on_device(20)])
        lists.update(change)
        return G.groot_adamw_tensors(**lists)
    whole, once = on_device(1000), on_device(300)
    bf16, codes = torch.bfloat16, torch.float8_e4m3fn
    for change in (dict(params=[whole[:300], whole[280:300]]), dict(params=[whole[10:310], whole[:20]]), dict(params=[once, once[100:120]]),
                   dict(m=[once, on_device(20)], v=[once, on_device(20)]), dict(params=[once, on_device(20)], master=[once, on_device(20)]),
                   dict(params=[once, on_device(20)], grads=[once, on_device(20)]), dict(params=[on_device(300), once[:20]], grads=[once, on_device(20)]),
                   dict(params=[on_device(300), once[299:300]], grads=[once, on_device(1)], m=[on_device(300), on_device(1)], v=[on_device(300), on_device(1)]),
                   dict(m=[on_device(300, dtype=codes), on_device(20, dtype=codes)], v=[on_device(300, dtype=codes), on_device(20, dtype=codes)],
                        m_scale=[once[:2], once[4:5]], v_scale=[once[2:4], once[4:5]])):
        with pytest.raises(ValueError, match="overlap"):
            make(**change)
    # neighbours, a gradient of two parameters, arrays of nothing
    t = make(params=[whole[:300], whole[300:320]], m=[whole[320:620], whole[980:]], v=[whole[640:940], whole[620:640]])
    make(grads=[once, once[:20]])
    make(params=[on_device(300), whole[5:5]], grads=[on_device(300), once[3:3]], m=[on_device(300), whole[5:5]], v=[on_device(300), whole[5:5]])
    before = t.array.copy()
    with pytest.raises(ValueError, match="overlap"):
        t.set_grads([whole.view(bf16)[:300], on_device(20, dtype=bf16)])
    assert t.grad_dtype == G.GROOT_F32 and (t.array == before).all()
