"""Host-side refusals of the calls that adapt a frozen layer: answered before anything would be launched, so they run
without a device.  Pointers are fakes that nothing dereferences."""
import ctypes
import types

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


SHAPE = B.make_shape(64, 256, 8, 512, 0, 2, 1)


def _balance(lib, shape=SHAPE, scores=P, idx=P, n_sel=P, off=P, n_seq=3, alpha=0.1, counts=P, coef=P, loss=P, st=P, ws=P,
             nb=BIG):
    return lib.moe_balance_loss(ctypes.byref(shape), scores, idx, n_sel, off, n_seq, alpha, counts, coef, loss, st, ws, nb, None)


@pytest.mark.parametrize("kw", [
    dict(scores=None), dict(idx=None), dict(counts=None), dict(coef=None), dict(loss=None), dict(st=None), dict(ws=None),
    dict(scores=ODD), dict(coef=ODD), dict(n_sel=P + 2), dict(off=P + 1), dict(off=None), dict(n_seq=0), dict(n_seq=-1),
    dict(n_seq=(1 << 20) + 1), dict(alpha=float("nan")), dict(alpha=float("inf")),
    dict(shape=B.make_shape(64, 256, 6, 512, 0, 2, 1)), dict(shape=B.make_shape(0, 256, 8, 512, 0, 2, 1)),
    dict(shape=B.make_shape((1 << 30) + 1, 256, 8, 512, 0, 1, 1))])
def test_balance_loss_refuses(lib, kw):
    assert _balance(lib, **kw) == B.MOE_ERR_ARG


def test_balance_loss_refuses_a_small_workspace(lib):
    need = B.moe_router_workspace_bytes(SHAPE, 3)
    assert need > 0 and _balance(lib, nb=need - 1) == B.MOE_ERR_WORKSPACE


def _gate(lib, shape=SHAPE, x=P, W=P, scores=P, idx=P, n_sel=P, d_top=P, coef=P, off=P, n_seq=3, d_logits=2 * P, dx=3 * P, dW=P,
          db=P, st=P, ws=P, nb=BIG):
    return lib.moe_gate_backward(ctypes.byref(shape), x, W, scores, idx, n_sel, d_top, coef, off, n_seq, d_logits, dx, dW, db, st,
                                 ws, nb, None)


@pytest.mark.parametrize("kw", [
    dict(scores=None), dict(d_top=None, coef=None), dict(idx=None), dict(x=None), dict(W=None), dict(st=None), dict(ws=None),
    dict(d_logits=None, dx=None, dW=None, db=None), dict(x=ODD), dict(W=ODD), dict(dx=ODD), dict(dW=ODD), dict(db=ODD),
    dict(d_top=ODD), dict(dx=P), dict(d_logits=P), dict(off=None), dict(n_seq=0), dict(n_sel=P + 1)])
def test_gate_backward_refuses(lib, kw):
    assert _gate(lib, **kw) == B.MOE_ERR_ARG


def test_gate_backward_refuses_a_small_workspace(lib):
    assert _gate(lib, nb=B.moe_router_workspace_bytes(SHAPE, 3) - 1) == B.MOE_ERR_WORKSPACE


def _combine(lib, shape=SHAPE, d_out=P, y=2 * P, pos=P, sc=P, n_sel=P, budget=128, ds=P, dy=3 * P):
    return lib.moe_combine_backward(ctypes.byref(shape), d_out, y, pos, sc, n_sel, budget, ds, dy, None)


@pytest.mark.parametrize("kw,status", [
    (dict(d_out=None), B.MOE_ERR_ARG), (dict(y=None), B.MOE_ERR_ARG), (dict(pos=None), B.MOE_ERR_ARG),
    (dict(n_sel=None), B.MOE_ERR_ARG), (dict(ds=None), B.MOE_ERR_ARG), (dict(sc=None), B.MOE_ERR_ARG),
    (dict(dy=2 * P), B.MOE_ERR_ARG), (dict(dy=P), B.MOE_ERR_ARG), (dict(dy=ODD), B.MOE_ERR_ARG), (dict(y=ODD), B.MOE_ERR_ARG),
    (dict(budget=-1), B.MOE_ERR_BUDGET), (dict(budget=129), B.MOE_ERR_BUDGET)])
def test_combine_backward_refuses(lib, kw, status):
    assert _combine(lib, **kw) == status


def test_combine_backward_refuses_more_pairs_than_positions(lib):
    assert _combine(lib, shape=B.make_shape(1 << 30, 256, 8, 512, 0, 2, 1)) == B.MOE_ERR_ARG


def test_router_workspace_is_zero_for_what_cannot_run(lib):
    assert B.moe_router_workspace_bytes(SHAPE, 0) == 0
    assert B.moe_router_workspace_bytes(SHAPE, (1 << 20) + 1) == 0
    assert B.moe_router_workspace_bytes(B.make_shape(64, 100, 8, 512, 0, 2, 1), 1) == 0
    assert B.moe_router_workspace_bytes(B.make_shape((1 << 30) + 1, 256, 8, 512, 0, 1, 1), 1) == 0
    with pytest.raises(B.MoeError):
        B.new_router_workspace(SHAPE, 0, device="cpu")


def test_binding_refuses_wrong_tensors(lib, monkeypatch):
    """dtype, size, contiguity and device of every tensor are looked at before the library is called."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)      # where CPU tensors say that they live
    monkeypatch.setattr(B, "_stream", lambda s=None: None)
    T, N, K = SHAPE.T, SHAPE.N, SHAPE.K_orig
    f = lambda *s: torch.zeros(*s)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    good = dict(scores=f(T, N), topk_idx=i(T, K), n_sel=i(T), seq_offsets=i(4), alpha=0.1, counts=i(3, N), coef=f(3, N), loss=f(1),
                dev_status=i(1), ws=torch.zeros(16, dtype=torch.uint8))
    bad = dict(scores=[f(T, N).double(), f(T, N + 4), f(N, T).t(), None], topk_idx=[i(T, K).long(), i(T, K + 1), None],
               n_sel=[i(T + 1), i(T).float()], counts=[i(2, N), None], coef=[f(3, N).half()], loss=[f(2)], dev_status=[i(2), None],
               seq_offsets=[i(1)], ws=[None])
    with pytest.raises(B.MoeError) as e:
        B.moe_balance_loss(SHAPE, **good)
    assert e.value.status == B.MOE_ERR_WORKSPACE                        # every tensor passed, the 16 bytes did not
    for name, values in bad.items():
        for v in values:
            with pytest.raises(B.MoeError) as e:
                B.moe_balance_loss(SHAPE, **{**good, name: v})
            assert e.value.status == B.MOE_ERR_ARG, name
    with pytest.raises(B.MoeError) as e:                                # a stream of another device
        B.moe_balance_loss(SHAPE, **good, stream=types.SimpleNamespace(device=torch.device("cuda", 3), cuda_stream=0))
    assert e.value.status == B.MOE_ERR_ARG


ASHAPE = B.make_adapter_shape(64, 256, 128, 4, 16)


def _linear(lib, shape=ASHAPE, x=P, W=P, A=P, Bm=P, scale=P, ids=P, y=2 * P, st=P, ws=P, nb=BIG):
    return lib.moe_adapter_linear(ctypes.byref(shape), x, W, A, Bm, scale, ids, y, st, ws, nb, None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(W=None), dict(A=None), dict(Bm=None), dict(scale=None), dict(ids=None), dict(y=None), dict(st=None),
    dict(ws=None), dict(x=ODD), dict(W=ODD), dict(A=ODD), dict(Bm=ODD), dict(y=ODD), dict(scale=P + 2), dict(ids=P + 1), dict(y=P)] + [
    dict(shape=B.make_adapter_shape(*v)) for v in ((0, 256, 128, 4, 16), (64, 250, 128, 4, 16), (64, 256, 124, 4, 16),
                                                   (64, 0, 128, 4, 16), (64, 256, 128, 0, 16), (64, 256, 128, 4, 12),
                                                   (64, 256, 128, 4, 136), (64, 256, 128, 4, 0), (64, 256, 128, 1 << 21, 16),
                                                   ((1 << 30) + 1, 256, 128, 4, 16), (64, (1 << 30) + 8, 128, 4, 16),
                                                   (64, 256, (1 << 30) + 8, 4, 16))])
def test_adapter_linear_refuses(lib, kw):
    assert _linear(lib, **kw) == B.MOE_ERR_ARG


def test_adapter_workspaces(lib):
    need = B.moe_adapter_workspace_bytes(ASHAPE)
    assert need > 0 and _linear(lib, nb=need - 1) == B.MOE_ERR_WORKSPACE
    bad = B.make_adapter_shape(64, 256, 128, 4, 16)
    bad.flags = 1
    assert B.moe_adapter_workspace_bytes(bad) == 0 and _linear(lib, shape=bad) == B.MOE_ERR_ARG
    s = B.make_shape(64, 256, 8, 512, 2, 2, 1)
    assert B.moe_shared_adapted_workspace_bytes(s, 4, 16) >= 64 * 2 * 512 * 2
    for args in ((B.make_shape(64, 256, 8, 512, 0, 2, 1), 4, 16), (s, 0, 16), (s, 4, 20)):
        assert B.moe_shared_adapted_workspace_bytes(*args) == 0
        with pytest.raises(B.MoeError):
            B.new_shared_adapted_workspace(*args, device="cpu")
    with pytest.raises(B.MoeError):
        B.new_adapter_workspace(bad, device="cpu")


@pytest.mark.parametrize("at", range(9))
def test_shared_ffn_adapted_refuses(lib, at):
    s = B.make_shape(64, 256, 8, 512, 2, 2, 1)

    def call(ptrs, shape=s, n=4, r=16, scale=P, ids=P, st=P, nb=BIG):
        x, W13, W2, A13, B13, A2, B2, y, ws = ptrs
        return lib.moe_shared_ffn_adapted(ctypes.byref(shape), n, r, x, W13, W2, A13, B13, A2, B2, scale, ids, y, st, ws, nb, None)

    good = [P] * 7 + [2 * P, P]
    for v in (None, ODD):
        assert call([v if i == at else g for i, g in enumerate(good)]) == B.MOE_ERR_ARG
    if at == 0:
        need = B.moe_shared_adapted_workspace_bytes(s, 4, 16)
        assert call(good, nb=need - 1) == B.MOE_ERR_WORKSPACE
        assert call([P] * 9) == B.MOE_ERR_ARG                                       # y_shared is x
        for kw in (dict(scale=None), dict(ids=None), dict(st=None), dict(n=0), dict(r=130), dict(r=4),
                   dict(shape=B.make_shape(64, 256, 8, 512, 0, 2, 1)), dict(shape=B.make_shape(64, 256, 8, 500, 2, 2, 1))):
            assert call(good, **kw) == B.MOE_ERR_ARG
