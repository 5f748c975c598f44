"""Host-side refusals of the calls for training the layer: answered before anything would be launched, so they run without a device.
Pointers are fakes that nothing dereferences."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2604_08133_b200 import binding as B

P, ODD = 1 << 20, (1 << 20) + 4
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return B.lib()


def _g(P_=100, K=64, M=128, E=8, flags=0):
    return B.MoeGroupedShape(P_, K, M, E, flags)


BAD_GROUPED = [_g(0), _g((1 << 30) + 1), _g(K=0), _g(K=12), _g(M=4), _g(M=20), _g(E=0), _g(E=129), _g(flags=4), _g(1 << 30, K=1 << 14),
               _g(K=1 << 20, M=1 << 20, E=64), _g(8, K=1 << 19, M=1 << 18, E=1)]


@pytest.mark.parametrize("name", ["moe_grouped_gemm", "moe_grouped_gemm_dx", "moe_grouped_gemm_dw"])
def test_products_refuse(lib, name):
    fn = getattr(lib, name)
    args = [P, 2 * P, 3 * P, 4 * P, P]
    for s in BAD_GROUPED:
        assert fn(ctypes.byref(s), *args, None) == B.MOE_ERR_ARG, (s.P, s.K, s.M, s.E, s.flags)
    assert fn(None, *args, None) == B.MOE_ERR_ARG
    s = _g()
    for i in range(5):
        assert fn(ctypes.byref(s), *args[:i], None, *args[i + 1:], None) == B.MOE_ERR_ARG, i
    for i in range(4):
        offset = i == (2 if name.endswith("dw") else 1)
        bad = args[i] + (2 if offset else 4)
        assert fn(ctypes.byref(s), *args[:i], bad, *args[i + 1:], None) == B.MOE_ERR_ARG, i
    assert fn(ctypes.byref(s), P, 2 * P, 3 * P, P, P, None) == B.MOE_ERR_ARG      # the output is an input
    other = 3 * P if not name.endswith("dw") else 2 * P
    assert fn(ctypes.byref(s), P, 2 * P, 3 * P, other, P, None) == B.MOE_ERR_ARG


def test_products_refuse_flags_that_are_not_theirs(lib):
    for name in ("moe_grouped_gemm", "moe_grouped_gemm_dx"):
        assert getattr(lib, name)(ctypes.byref(_g(flags=1)), P, 2 * P, 3 * P, 4 * P, P, None) == B.MOE_ERR_ARG
    assert lib.moe_grouped_gemm_dw(ctypes.byref(_g(flags=2)), P, 2 * P, 3 * P, 4 * P, P, None) == B.MOE_ERR_ARG   # bf16 sums are not added to


SHAPE = B.make_shape(64, 256, 8, 512, 0, 2, 1)


def _ffn(lib, shape=SHAPE, x=P, tok=P, off=P, budget=64, W13=P, W2=P, dy=P, dx=2 * P, dW13=3 * P, dW2=4 * P, st=P, ws=P, nb=BIG):
    return lib.moe_grouped_ffn_backward(ctypes.byref(shape), x, tok, off, budget, W13, W2, dy, dx, dW13, dW2, st, ws, nb, None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(off=None), dict(W13=None), dict(W2=None), dict(dy=None), dict(st=None), dict(ws=None), dict(dx=None, dW13=None, dW2=None),
    dict(x=ODD), dict(W13=ODD), dict(W2=ODD), dict(dy=ODD), dict(dx=ODD), dict(dW13=ODD), dict(dW2=ODD), dict(ws=ODD), dict(tok=P + 2),
    dict(off=P + 1), dict(dx=P), dict(dW13=P), dict(dW2=P), dict(shape=B.make_shape(64, 200, 8, 512, 0, 2, 1))])
def test_experts_backward_refuses(lib, kw):
    assert _ffn(lib, **kw) == B.MOE_ERR_ARG


def test_experts_backward_refuses_budgets_and_workspaces(lib):
    assert _ffn(lib, budget=-1) == B.MOE_ERR_BUDGET and _ffn(lib, budget=129) == B.MOE_ERR_BUDGET
    need = B.moe_ffn_backward_workspace_bytes(SHAPE, 64)
    assert need >= 64 * (256 + 3 * 512) * 2 and _ffn(lib, nb=need - 1) == B.MOE_ERR_WORKSPACE
    assert B.moe_ffn_backward_workspace_bytes(SHAPE, 129) == 0 and B.moe_ffn_backward_workspace_bytes(SHAPE, -1) == 0
    assert 0 < B.moe_ffn_backward_workspace_bytes(SHAPE, 0) < need


SHARED = B.make_shape(64, 256, 8, 512, 2, 2, 1)


def _shared(lib, shape=SHARED, x=P, W13=P, W2=P, dy=P, dx=2 * P, dW13=3 * P, dW2=4 * P, st=P, ws=P, nb=BIG):
    return lib.moe_shared_ffn_backward(ctypes.byref(shape), x, W13, W2, dy, dx, dW13, dW2, st, ws, nb, None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(W13=None), dict(W2=None), dict(dy=None), dict(st=None), dict(ws=None), dict(dx=None, dW13=None, dW2=None), dict(x=ODD),
    dict(W13=ODD), dict(W2=ODD), dict(dy=ODD), dict(dx=ODD), dict(dW13=ODD), dict(dW2=ODD), dict(ws=ODD), dict(dx=P), dict(dW13=P), dict(dW2=P),
    dict(shape=SHAPE), dict(shape=B.make_shape(64, 200, 8, 512, 2, 2, 1)), dict(shape=B.make_shape((1 << 30) + 1, 256, 8, 512, 2, 1, 1))])
def test_shared_backward_refuses(lib, kw):
    assert _shared(lib, **kw) == B.MOE_ERR_ARG


def test_shared_backward_refuses_a_small_workspace(lib):
    need = B.moe_shared_ffn_backward_workspace_bytes(SHARED)
    assert need >= 64 * 2 * 3 * 512 * 2 and _shared(lib, nb=need - 1) == B.MOE_ERR_WORKSPACE
    assert B.moe_shared_ffn_backward_workspace_bytes(SHAPE) == 0


def _n(T=64, H=256, gate=1, eps=1e-6, flags=0):
    return B.MoeNormShape(T, H, gate, eps, flags)


BAD_NORM = [_n(0), _n((1 << 30) + 1), _n(H=0), _n(H=12), _n(H=8200), _n(gate=2), _n(gate=-1), _n(eps=0.0), _n(eps=-1.0), _n(eps=float("inf")),
            _n(eps=float("nan")), _n(flags=2)]


def _norm(lib, shape=None, r=P, y=2 * P, wp=P, gate=P + 2, scale=P, wn=P, ro=3 * P, no=4 * P):
    return lib.moe_block_norm(ctypes.byref(shape or _n()), r, y, wp, gate, scale, wn, ro, no, None)


@pytest.mark.parametrize("kw", [dict(shape=s) for s in BAD_NORM] + [
    dict(r=None), dict(y=None), dict(ro=None), dict(ro=None, no=None), dict(gate=None), dict(shape=_n(gate=0)), dict(r=ODD), dict(y=ODD),
    dict(wp=ODD), dict(wn=ODD), dict(ro=ODD), dict(no=ODD), dict(scale=P + 2), dict(gate=P + 1), dict(shape=_n(gate=256)), dict(no=3 * P),
    dict(no=P), dict(ro=2 * P), dict(y=None, ro=None, no=None)])
def test_block_norm_refuses(lib, kw):
    assert _norm(lib, **kw) == B.MOE_ERR_ARG


def _norm_b(lib, shape=None, r=P, y=2 * P, wp=P, gate=6 * P, scale=P, wn=P, dn=3 * P, dro=4 * P, dr=5 * P, dy=7 * P, dg=8 * P, dwp=9 * P,
            dwn=10 * P, ds=11 * P, ws=P, nb=BIG):
    return lib.moe_block_norm_backward(ctypes.byref(shape or _n()), r, y, wp, gate, scale, wn, dn, dro, dr, dy, dg, dwp, dwn, ds, ws, nb, None)


@pytest.mark.parametrize("kw", [dict(shape=s) for s in BAD_NORM] + [
    dict(r=None), dict(dn=None, dro=None), dict(gate=None), dict(shape=_n(gate=0)), dict(y=None), dict(dn=None), dict(ws=None),
    dict(dr=None, dy=None, dg=None, dwp=None, dwn=None, ds=None), dict(r=ODD), dict(y=ODD), dict(dn=ODD), dict(dro=ODD), dict(dr=ODD),
    dict(dy=ODD), dict(dwp=ODD), dict(dwn=ODD), dict(ws=ODD), dict(ds=11 * P + 2), dict(dg=8 * P + 1), dict(dr=P), dict(dr=2 * P), dict(dy=P),
    dict(dy=3 * P), dict(dg=6 * P), dict(dwp=P), dict(ds=4 * P)])
def test_block_norm_backward_refuses(lib, kw):
    assert _norm_b(lib, **kw) == B.MOE_ERR_ARG


OUT = 13 * P


@pytest.mark.parametrize("call,names", [(_ffn, ("dx", "dW13", "dW2", "ws")), (_shared, ("dx", "dW13", "dW2", "ws")),
                                        (_norm_b, ("dr", "dy", "dg", "dwp", "dwn", "ds", "ws"))])
def test_backward_passes_refuse_two_outputs_that_are_one(lib, call, names):
    for i, a in enumerate(names):
        for b in names[:i]:
            assert call(lib, **{a: OUT, b: OUT, "nb": 0}) == B.MOE_ERR_ARG, (a, b)
        assert call(lib, **{a: OUT, "nb": 0}) == B.MOE_ERR_WORKSPACE, a        # by itself it is not what is wrong


def test_block_norm_backward_refuses_a_small_workspace(lib):
    need = B.moe_norm_workspace_bytes(_n())
    assert need > 0 and _norm_b(lib, nb=need - 1) == B.MOE_ERR_WORKSPACE
    assert all(B.moe_norm_workspace_bytes(s) == 0 for s in BAD_NORM)


def _entry(**kw):
    e = dict(param=P, grad=2 * P, m=3 * P, v=4 * P, m_scale=None, v_scale=None, copy=None, n=1000, weight_decay=0.1, flags=0)
    e.update(kw)
    return (B.MoeAdamwTensor * 1)(B.MoeAdamwTensor(*[e[k] for k in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy", "n",
                                                                   "weight_decay", "flags")]))


def _adam(lib, entry=None, count=1, b1=0.9, b2=0.999, eps=1e-8, hyper=P, st=P):
    return lib.moe_adamw_step(entry if entry is not None else _entry(), count, b1, b2, eps, hyper, st, None)


@pytest.mark.parametrize("kw", [
    dict(count=0), dict(count=-1), dict(count=(1 << 20) + 1), dict(b1=1.0), dict(b1=-0.1), dict(b1=float("nan")), dict(b2=1.0), dict(b2=-1.0),
    dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=float("nan")), dict(eps=float("inf")), dict(hyper=None), dict(st=None),
    dict(hyper=P + 2)])
def test_adamw_step_refuses(lib, kw):
    assert _adam(lib, **kw) == B.MOE_ERR_ARG


@pytest.mark.parametrize("kw", [
    dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=0), dict(n=-5), dict(n=1 << 60), dict(param=ODD), dict(grad=ODD),
    dict(m=ODD), dict(v=ODD), dict(copy=ODD), dict(flags=8), dict(flags=4), dict(flags=4, m_scale=P), dict(flags=4, m_scale=P, v_scale=P + 2),
    dict(weight_decay=float("nan")), dict(weight_decay=float("inf")), dict(grad=P)])
def test_adamw_step_refuses_entries(lib, kw):
    assert _adam(lib, entry=_entry(**kw)) == B.MOE_ERR_ARG


def test_adamw_states_refuse(lib):
    good = dict(flags=4, m_scale=P, v_scale=P)
    one = lambda v: (ctypes.c_void_p * 1)(v)
    for e, m, v in ((_entry(), one(P), one(2 * P)), (_entry(**good), None, one(P)), (_entry(**good), one(P), None),
                    (_entry(**good), one(None), one(P)), (_entry(**good), one(ODD), one(P)), (_entry(**good), one(P), one(P)),
                    (_entry(**dict(good, m_scale=None)), one(P), one(2 * P))):
        assert lib.moe_adamw_states_read(e, 1, m, v, None) == B.MOE_ERR_ARG
        assert lib.moe_adamw_states_write(e, 1, m, v, P, None) == B.MOE_ERR_ARG
    assert lib.moe_adamw_states_write(_entry(**good), 1, one(P), one(2 * P), None, None) == B.MOE_ERR_ARG


def test_the_list_of_tensors_refuses_what_is_not_on_a_device():
    for items in ([], [dict()], [dict(param=torch.zeros(8), grad=torch.zeros(8), m=torch.zeros(8), v=torch.zeros(8))]):
        with pytest.raises(B.MoeError) as e:
            B.make_adamw_tensors(items)
        assert e.value.status == B.MOE_ERR_ARG
