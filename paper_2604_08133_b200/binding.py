"""ctypes binding of liballocmoe.so: the same names as include/allocmoe.h, argument
marshalling only.  torch supplies device memory and streams; every step of the path runs in
the library's kernels.  There is no fallback: a missing library is an error."""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# ALLOCMOE_LIB selects another build of the same library (the checked build, see build.py)
LIB_PATH = os.environ.get("ALLOCMOE_LIB") or os.path.join(_PKG, "liballocmoe.so")

MOE_OK, MOE_ERR_ARG, MOE_ERR_BUDGET, MOE_ERR_WORKSPACE, MOE_ERR_CUDA, MOE_ERR_NONFINITE, MOE_ERR_TIMEOUT = range(7)

EXPORTS = ("moe_status_string", "moe_workspace_bytes", "moe_gate", "alloc_t_select", "moe_permute",
           "moe_grouped_ffn", "moe_shared_ffn", "moe_combine", "moe_layer_forward", "moe_layer_intermediates",
           "moe_rmsnorm", "moe_profile_enable", "moe_profile_read", "moe_permute_static", "moe_route", "alloc_l_solve",
           "moe_layer_forward_routed", "moe_selftest_wait_timeout", "moe_select_top_p", "moe_select_rel_threshold",
           "moe_router_workspace_bytes", "moe_balance_loss", "moe_gate_backward", "moe_combine_backward",
           "moe_adapter_workspace_bytes", "moe_adapter_linear", "moe_shared_adapted_workspace_bytes",
           "moe_shared_ffn_adapted", "moe_grouped_gemm", "moe_grouped_gemm_dx", "moe_grouped_gemm_dw",
           "moe_ffn_backward_workspace_bytes", "moe_grouped_ffn_backward", "moe_block_norm", "moe_norm_workspace_bytes",
           "moe_block_norm_backward", "moe_shared_ffn_backward_workspace_bytes", "moe_shared_ffn_backward", "moe_adamw_step", "moe_adamw_states_read", "moe_adamw_states_write")
PROFILE_STAGES = ("gate", "route", "gather", "ffn_gemm1", "ffn_gemm2", "combine")


class MoeShape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("I", ctypes.c_int32),
                ("S", ctypes.c_int32), ("K_orig", ctypes.c_int32), ("K_base", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class MoeAdapterShape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("K", ctypes.c_int32), ("M", ctypes.c_int32), ("n_adapters", ctypes.c_int32),
                ("rank", ctypes.c_int32), ("flags", ctypes.c_uint32)]


MOE_GROUPED_DW_FP32, MOE_GROUPED_DW_ADD = 1, 2
MOE_NORM_Y_AS_IS = 1
MOE_ADAMW_PARAM_BF16, MOE_ADAMW_GRAD_BF16, MOE_ADAMW_STATE8 = 1, 2, 4
ADAMW_BLOCK = 256   # elements of an 8-bit state that share a scale


class MoeGroupedShape(ctypes.Structure):
    _fields_ = [("P", ctypes.c_int32), ("K", ctypes.c_int32), ("M", ctypes.c_int32), ("E", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class MoeNormShape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("gate_cols", ctypes.c_int32), ("eps", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


class MoeAdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("weight_decay", ctypes.c_float), ("flags", ctypes.c_uint32)]


class MoeError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {status_string(status)} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the C-ABI library (built by `python -m paper_2604_08133_b200.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_08133_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
        sp = ctypes.POINTER(MoeShape)
        L.moe_status_string.restype = ctypes.c_char_p
        L.moe_status_string.argtypes = [ctypes.c_int]
        L.moe_workspace_bytes.restype = sz
        L.moe_workspace_bytes.argtypes = [sp, i64]
        L.moe_router_workspace_bytes.restype = sz
        L.moe_router_workspace_bytes.argtypes = [sp, ctypes.c_int32]
        i32, f32 = ctypes.c_int32, ctypes.c_float
        ap = ctypes.POINTER(MoeAdapterShape)
        L.moe_adapter_workspace_bytes.restype = sz
        L.moe_adapter_workspace_bytes.argtypes = [ap]
        L.moe_shared_adapted_workspace_bytes.restype = sz
        L.moe_shared_adapted_workspace_bytes.argtypes = [sp, i32, i32]
        gp, np_, tp = ctypes.POINTER(MoeGroupedShape), ctypes.POINTER(MoeNormShape), ctypes.POINTER(MoeAdamwTensor)
        f64 = ctypes.c_double
        L.moe_ffn_backward_workspace_bytes.restype = sz
        L.moe_ffn_backward_workspace_bytes.argtypes = [sp, i64]
        L.moe_shared_ffn_backward_workspace_bytes.restype = sz
        L.moe_shared_ffn_backward_workspace_bytes.argtypes = [sp]
        L.moe_norm_workspace_bytes.restype = sz
        L.moe_norm_workspace_bytes.argtypes = [np_]
        sigs = {
            "moe_balance_loss": [sp, vp, vp, vp, vp, i32, f32, vp, vp, vp, vp, vp, sz, vp],
            "moe_gate_backward": [sp] + [vp] * 8 + [i32] + [vp] * 6 + [sz, vp],
            "moe_adapter_linear": [ap] + [vp] * 9 + [sz, vp],
            "moe_shared_ffn_adapted": [sp, i32, i32] + [vp] * 12 + [sz, vp],
            "moe_combine_backward": [sp, vp, vp, vp, vp, vp, i64, vp, vp, vp],
            "moe_grouped_gemm": [gp] + [vp] * 6,
            "moe_grouped_gemm_dx": [gp] + [vp] * 6,
            "moe_grouped_gemm_dw": [gp] + [vp] * 6,
            "moe_grouped_ffn_backward": [sp, vp, vp, vp, i64] + [vp] * 8 + [sz, vp],
            "moe_shared_ffn_backward": [sp] + [vp] * 9 + [sz, vp],
            "moe_block_norm": [np_] + [vp] * 9,
            "moe_block_norm_backward": [np_] + [vp] * 15 + [sz, vp],
            "moe_adamw_step": [tp, i32, f64, f64, f64, vp, vp, vp],
            "moe_adamw_states_read": [tp, i32, vp, vp, vp],
            "moe_adamw_states_write": [tp, i32, vp, vp, vp, vp],
            "moe_gate": [sp, vp, vp, vp, vp, vp, vp, vp],
            "alloc_t_select": [sp, vp, i64, vp, vp, vp, sz, vp],
            "moe_permute": [sp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "moe_permute_static": [sp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp],
            "moe_route": [sp, vp, vp, i64, vp, vp, vp, vp, vp, vp, vp],
            "moe_grouped_ffn": [sp, vp, vp, vp, i64, vp, vp, vp, vp, vp, sz, vp],
            "moe_layer_forward_routed": [sp, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "moe_selftest_wait_timeout": [sp, vp, i64, vp, vp, i64, vp, vp, sz, vp],
            "moe_select_top_p": [sp, vp, ctypes.c_float, vp, vp, vp, vp],
            "moe_select_rel_threshold": [sp, vp, ctypes.c_float, vp, vp, vp, vp],
            "moe_shared_ffn": [sp, vp, vp, vp, vp, vp, vp, sz, vp],
            "moe_combine": [sp, vp, vp, vp, vp, vp, vp, vp],
            "moe_layer_forward": [sp, vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, sz, vp],
            "moe_rmsnorm": [sp, vp, vp, vp],
            "moe_layer_intermediates": [sp, i64, vp, sz] + [ctypes.POINTER(vp)] * 7,
            "moe_profile_enable": [ctypes.c_int32],
            "moe_profile_read": [ctypes.POINTER(ctypes.c_float)],
        }
        L.alloc_l_solve.restype = ctypes.c_int
        L.alloc_l_solve.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.c_int32, ctypes.c_int32, i64,
                                    ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_double)]
        for name, argtypes in sigs.items():
            fn = getattr(L, name)
            fn.restype = ctypes.c_int
            fn.argtypes = argtypes
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().moe_status_string(int(status)).decode()


def make_shape(T, H, N, I, S, K_orig, K_base) -> MoeShape:
    return MoeShape(int(T), int(H), int(N), int(I), int(S), int(K_orig), int(K_base), 0)


def shape_of(cfg) -> MoeShape:
    return make_shape(cfg.T, cfg.H, cfg.N, cfg.I, cfg.S, cfg.K_orig, cfg.K_base)


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous()
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    # the raw handle of the current stream; building a torch.cuda.Stream object for it would cost 3 us a call
    if stream is None:
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def _check(fn: str, st: int):
    if st != MOE_OK:
        raise MoeError(fn, st)


def moe_workspace_bytes(shape: MoeShape, budget_max: int) -> int:
    return int(lib().moe_workspace_bytes(ctypes.byref(shape), int(budget_max)))


def new_workspace(shape: MoeShape, budget_max: int, device="cuda") -> torch.Tensor:
    n = moe_workspace_bytes(shape, budget_max)
    if n == 0:
        raise MoeError("moe_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_gate(shape, x, W_gate, gate_bias, scores, topk_idx, topk_score, stream=None):
    _check("moe_gate", lib().moe_gate(ctypes.byref(shape), _p(x), _p(W_gate), _p(gate_bias), _p(scores),
                                      _p(topk_idx), _p(topk_score), _stream(stream)))


def alloc_t_select(shape, topk_score, budget, n_sel, dev_status, ws, stream=None):
    _check("alloc_t_select", lib().alloc_t_select(ctypes.byref(shape), _p(topk_score), int(budget), _p(n_sel),
                                                  _p(dev_status), _p(ws), ws.numel() if ws is not None else 0,
                                                  _stream(stream)))


def moe_permute(shape, x, topk_idx, topk_score, n_sel, budget, expert_offsets, perm_token, perm_weight, pair_pos,
                x_perm, dev_status, ws, stream=None):
    _check("moe_permute", lib().moe_permute(ctypes.byref(shape), _p(x), _p(topk_idx), _p(topk_score), _p(n_sel),
                                            int(budget), _p(expert_offsets), _p(perm_token), _p(perm_weight),
                                            _p(pair_pos), _p(x_perm), _p(dev_status), _p(ws), ws.numel(),
                                            _stream(stream)))


def alloc_l_solve(S, B: int):
    """Alloc-L (Eq. 3-6): the optimal per-layer K for a sensitivity matrix S [L, K_orig] (any array-like of floats)
    under the global budget B.  Returns (list of K_i, total cost).  Host only."""
    rows = [[float(v) for v in r] for r in S]
    Lr, K = len(rows), len(rows[0])
    flat = (ctypes.c_double * (Lr * K))(*[v for r in rows for v in r])
    out = (ctypes.c_int32 * Lr)()
    cost = ctypes.c_double(0.0)
    _check("alloc_l_solve", lib().alloc_l_solve(flat, Lr, K, int(B), out, ctypes.byref(cost)))
    return list(out), float(cost.value)


def moe_route(shape, topk_idx, topk_score, budget, n_sel, expert_offsets, perm_token, perm_weight, pair_pos, dev_status,
              stream=None):
    """alloc_t_select + the list-building part of moe_permute in one launch (T <= 8192)."""
    _check("moe_route", lib().moe_route(ctypes.byref(shape), _p(topk_idx), _p(topk_score), int(budget), _p(n_sel),
                                        _p(expert_offsets), _p(perm_token), _p(perm_weight), _p(pair_pos),
                                        _p(dev_status), _stream(stream)))


def moe_permute_static(shape, x, topk_idx, topk_score, n_sel, budget, expert_offsets, perm_token, perm_weight, pair_pos,
                       x_perm, dev_status, stream=None):
    """moe_permute without a workspace argument, for callers that cannot allocate device memory:
    the scratch is a fixed array inside the library (N * ceil(T/32) <= 65536)."""
    _check("moe_permute_static", lib().moe_permute_static(ctypes.byref(shape), _p(x), _p(topk_idx), _p(topk_score),
                                                          _p(n_sel), int(budget), _p(expert_offsets), _p(perm_token),
                                                          _p(perm_weight), _p(pair_pos), _p(x_perm), _p(dev_status),
                                                          _stream(stream)))


def moe_grouped_ffn(shape, x_or_xperm, perm_token, expert_offsets, budget, W13, W2, y_perm, dev_status, ws, stream=None):
    """perm_token None: x_or_xperm is x_perm [budget,H]; else it is x [T,H] and row p is x[perm_token[p]]."""
    _check("moe_grouped_ffn", lib().moe_grouped_ffn(ctypes.byref(shape), _p(x_or_xperm), _p(perm_token),
                                                    _p(expert_offsets), int(budget), _p(W13), _p(W2), _p(y_perm),
                                                    _p(dev_status), _p(ws), ws.numel(), _stream(stream)))


def moe_shared_ffn(shape, x, Wsh13, Wsh2, y_shared, dev_status, ws, stream=None):
    _check("moe_shared_ffn", lib().moe_shared_ffn(ctypes.byref(shape), _p(x), _p(Wsh13), _p(Wsh2), _p(y_shared),
                                                  _p(dev_status), _p(ws), ws.numel(), _stream(stream)))


def moe_combine(shape, y_perm, pair_pos, topk_score, n_sel, y_shared, out, stream=None):
    _check("moe_combine", lib().moe_combine(ctypes.byref(shape), _p(y_perm), _p(pair_pos), _p(topk_score), _p(n_sel),
                                            _p(y_shared), _p(out), _stream(stream)))


def moe_layer_forward(shape, x, W_gate, gate_bias, W13, W2, Wsh13, Wsh2, budget, out, dev_status, ws,
                      residual: Optional[torch.Tensor] = None, stream=None):
    _check("moe_layer_forward", lib().moe_layer_forward(ctypes.byref(shape), _p(x), _p(W_gate), _p(gate_bias), _p(W13),
                                                        _p(W2), _p(Wsh13), _p(Wsh2), int(budget), _p(residual),
                                                        _p(out), _p(dev_status), _p(ws), ws.numel(), _stream(stream)))


def moe_layer_forward_routed(shape, x, topk_idx, topk_score, n_sel, budget_max, budget_hint, W13, W2, Wsh13, Wsh2, out,
                             dev_status, ws, residual: Optional[torch.Tensor] = None, stream=None):
    """Permutation, experts and combine for a selection the caller holds (n_sel on the device)."""
    _check("moe_layer_forward_routed",
           lib().moe_layer_forward_routed(ctypes.byref(shape), _p(x), _p(topk_idx), _p(topk_score), _p(n_sel),
                                          int(budget_max), int(budget_hint), _p(W13), _p(W2), _p(Wsh13), _p(Wsh2),
                                          _p(residual), _p(out), _p(dev_status), _p(ws), ws.numel(), _stream(stream)))


def moe_selftest_wait_timeout(shape, expert_offsets, budget, W2, y_perm, wait_limit_clk, dev_status, ws, stream=None):
    """Launches expert GEMM-2 alone with a short wait limit: its bounded waits run out (see the header)."""
    _check("moe_selftest_wait_timeout",
           lib().moe_selftest_wait_timeout(ctypes.byref(shape), _p(expert_offsets), int(budget), _p(W2), _p(y_perm),
                                           int(wait_limit_clk), _p(dev_status), _p(ws), ws.numel(), _stream(stream)))


def moe_select_top_p(shape, topk_score, P, n_sel, total, dev_status, stream=None):
    """Top-P count per token (the Dynamic-MoE baseline); `total` (device int32 [1] or None) accumulates sum n_sel."""
    _check("moe_select_top_p", lib().moe_select_top_p(ctypes.byref(shape), _p(topk_score), float(P), _p(n_sel),
                                                      _p(total), _p(dev_status), _stream(stream)))


def moe_select_rel_threshold(shape, topk_score, beta, n_sel, total, dev_status, stream=None):
    """Skipping relative to the top-1 score (the NAEE baseline extended to Top-K)."""
    _check("moe_select_rel_threshold",
           lib().moe_select_rel_threshold(ctypes.byref(shape), _p(topk_score), float(beta), _p(n_sel), _p(total),
                                          _p(dev_status), _stream(stream)))


# The calls below check what a C entry point cannot see (dtype, size, contiguity, device) and answer with the status
# that the library gives for a bad pointer or shape.
def _arg(fn: str, name: str, t: Optional[torch.Tensor], dtype, numel: int, dev: int, optional: bool = False):
    if t is None:
        if optional:
            return None
        raise MoeError(f"{fn}: {name} is missing", MOE_ERR_ARG)
    if t.dtype is not dtype or t.numel() != numel or t.get_device() != dev or not t.is_contiguous():
        raise MoeError(f"{fn}: {name} must be a contiguous {dtype} tensor of {numel} elements on cuda:{dev}", MOE_ERR_ARG)
    return t.data_ptr()


def _device(fn: str, stream) -> int:
    """The current device, on which the library launches; a stream of another one is refused."""
    dev = torch.cuda.current_device()
    if stream is not None and stream.device.index != dev:
        raise MoeError(f"{fn}: the stream belongs to {stream.device}, the current device is cuda:{dev}", MOE_ERR_ARG)
    return dev


def _handle(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _ws(fn: str, ws: Optional[torch.Tensor], dev: int):
    if ws is None or ws.get_device() != dev or not ws.is_contiguous():
        raise MoeError(f"{fn}: ws must be a contiguous tensor on cuda:{dev}", MOE_ERR_ARG)
    return ws.data_ptr(), ws.numel() * ws.element_size()


def moe_router_workspace_bytes(shape: MoeShape, n_seq: int = 1) -> int:
    return int(lib().moe_router_workspace_bytes(ctypes.byref(shape), int(n_seq)))


def new_router_workspace(shape: MoeShape, n_seq: int = 1, device="cuda") -> torch.Tensor:
    """Scratch for moe_balance_loss and moe_gate_backward with up to n_seq packed sequences."""
    n = moe_router_workspace_bytes(shape, n_seq)
    if n == 0:
        raise MoeError("moe_router_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def _n_seq(fn: str, seq_offsets: Optional[torch.Tensor]) -> int:
    n = 1 if seq_offsets is None else seq_offsets.numel() - 1
    if n < 1:
        raise MoeError(f"{fn}: seq_offsets needs at least two entries", MOE_ERR_ARG)
    return n


def moe_balance_loss(shape, scores, topk_idx, n_sel, seq_offsets, alpha, counts, coef, loss, dev_status, ws, stream=None):
    """Balance loss over the kept pairs, the per-expert counts behind it [n_seq, N] and its derivative with respect to
    the scores of each sequence, coef [n_seq, N] (for moe_gate_backward).  n_sel None: all K_orig columns are kept;
    seq_offsets None: one sequence of all T rows, else int32 [n_seq + 1]."""
    fn = "moe_balance_loss"
    dev, b = _device(fn, stream), _n_seq(fn, seq_offsets)
    i32, f32, T, N = torch.int32, torch.float32, shape.T, shape.N
    w, nw = _ws(fn, ws, dev)
    _check(fn, lib().moe_balance_loss(
        ctypes.byref(shape), _arg(fn, "scores", scores, f32, T * N, dev),
        _arg(fn, "topk_idx", topk_idx, i32, T * shape.K_orig, dev), _arg(fn, "n_sel", n_sel, i32, T, dev, True),
        _arg(fn, "seq_offsets", seq_offsets, i32, b + 1, dev, True), b, alpha,
        _arg(fn, "counts", counts, i32, b * N, dev), _arg(fn, "coef", coef, f32, b * N, dev),
        _arg(fn, "loss", loss, f32, 1, dev), _arg(fn, "dev_status", dev_status, i32, 1, dev), w, nw, _stream(stream)))


def moe_gate_backward(shape, x, W_gate, scores, topk_idx, n_sel, d_topk_score, coef, seq_offsets, d_logits, dx, dW_gate, d_bias,
                      dev_status, ws, stream=None):
    """Backward pass of moe_gate from the gradients of the kept scores (d_topk_score, or None) and the balance loss (coef,
    or None).  Outputs d_logits fp32 [T,N], dx bf16 [T,H], dW_gate fp32 [H,N], d_bias fp32 [N]: None is not computed.  x is
    needed for dW_gate only, W_gate for dx only, topk_idx for d_topk_score only."""
    fn = "moe_gate_backward"
    dev, b = _device(fn, stream), _n_seq(fn, seq_offsets)
    i32, f32, bf, T, N, H = torch.int32, torch.float32, torch.bfloat16, shape.T, shape.N, shape.H
    w, nw = _ws(fn, ws, dev)
    _check(fn, lib().moe_gate_backward(
        ctypes.byref(shape), _arg(fn, "x", x, bf, T * H, dev, True), _arg(fn, "W_gate", W_gate, bf, H * N, dev, True),
        _arg(fn, "scores", scores, f32, T * N, dev), _arg(fn, "topk_idx", topk_idx, i32, T * shape.K_orig, dev, True),
        _arg(fn, "n_sel", n_sel, i32, T, dev, True),
        _arg(fn, "d_topk_score", d_topk_score, f32, T * shape.K_orig, dev, True),
        _arg(fn, "coef", coef, f32, b * N, dev, True), _arg(fn, "seq_offsets", seq_offsets, i32, b + 1, dev, True), b,
        _arg(fn, "d_logits", d_logits, f32, T * N, dev, True), _arg(fn, "dx", dx, bf, T * H, dev, True),
        _arg(fn, "dW_gate", dW_gate, f32, H * N, dev, True), _arg(fn, "d_bias", d_bias, f32, N, dev, True),
        _arg(fn, "dev_status", dev_status, i32, 1, dev), w, nw, _stream(stream)))


def moe_combine_backward(shape, d_out, y_perm, pair_pos, topk_score, n_sel, budget, d_topk_score, d_y_perm, stream=None):
    """Gradients of Eq. 2's weighted sum with respect to the routing scores (fp32 [T, K_orig]) and, unless d_y_perm is
    None, the experts' rows (bf16 [budget, H])."""
    fn = "moe_combine_backward"
    dev, budget = _device(fn, stream), int(budget)
    i32, f32, bf, TK, H = torch.int32, torch.float32, torch.bfloat16, shape.T * shape.K_orig, shape.H
    _check(fn, lib().moe_combine_backward(
        ctypes.byref(shape), _arg(fn, "d_out", d_out, bf, shape.T * H, dev), _arg(fn, "y_perm", y_perm, bf, budget * H, dev),
        _arg(fn, "pair_pos", pair_pos, i32, TK, dev), _arg(fn, "topk_score", topk_score, f32, TK, dev, d_y_perm is None),
        _arg(fn, "n_sel", n_sel, i32, shape.T, dev), budget, _arg(fn, "d_topk_score", d_topk_score, f32, TK, dev),
        _arg(fn, "d_y_perm", d_y_perm, bf, budget * H, dev, True), _stream(stream)))


def make_adapter_shape(T, K, M, n_adapters, rank) -> MoeAdapterShape:
    return MoeAdapterShape(int(T), int(K), int(M), int(n_adapters), int(rank), 0)


def moe_adapter_workspace_bytes(ashape: MoeAdapterShape) -> int:
    return int(lib().moe_adapter_workspace_bytes(ctypes.byref(ashape)))


def new_adapter_workspace(ashape: MoeAdapterShape, device="cuda") -> torch.Tensor:
    n = moe_adapter_workspace_bytes(ashape)
    if n == 0:
        raise MoeError("moe_adapter_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_shared_adapted_workspace_bytes(shape: MoeShape, n_adapters: int, rank: int) -> int:
    return int(lib().moe_shared_adapted_workspace_bytes(ctypes.byref(shape), int(n_adapters), int(rank)))


def new_shared_adapted_workspace(shape: MoeShape, n_adapters: int, rank: int, device="cuda") -> torch.Tensor:
    n = moe_shared_adapted_workspace_bytes(shape, n_adapters, rank)
    if n == 0:
        raise MoeError("moe_shared_adapted_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_adapter_linear(ashape, x, W, A, B, scale, adapter_id, y, dev_status, ws, stream=None):
    """y[t] = x[t] W^T + scale[a] (x[t] A_a^T) B_a^T with a = adapter_id[t] (negative: no adapter).
    x [T,K], W [M,K], A [n,rank,K], B [n,M,rank], y [T,M] bf16; scale fp32 [n]; adapter_id int32 [T]."""
    fn = "moe_adapter_linear"
    dev = _device(fn, stream)
    i32, f32, bf = torch.int32, torch.float32, torch.bfloat16
    T, K, M, n, r = ashape.T, ashape.K, ashape.M, ashape.n_adapters, ashape.rank
    w, nw = _ws(fn, ws, dev)
    _check(fn, lib().moe_adapter_linear(
        ctypes.byref(ashape), _arg(fn, "x", x, bf, T * K, dev), _arg(fn, "W", W, bf, M * K, dev),
        _arg(fn, "A", A, bf, n * r * K, dev), _arg(fn, "B", B, bf, n * M * r, dev), _arg(fn, "scale", scale, f32, n, dev),
        _arg(fn, "adapter_id", adapter_id, i32, T, dev), _arg(fn, "y", y, bf, T * M, dev),
        _arg(fn, "dev_status", dev_status, i32, 1, dev), w, nw, _stream(stream)))


def moe_shared_ffn_adapted(shape, x, Wsh13, Wsh2, A13, B13, A2, B2, scale, adapter_id, y_shared, dev_status, ws, stream=None):
    """moe_shared_ffn with a low-rank adapter per token beside both projections: A13 [n,rank,H], B13 [n,S*2I,rank],
    A2 [n,rank,S*I], B2 [n,H,rank].  The number of adapters and the rank are those of A13."""
    fn = "moe_shared_ffn_adapted"
    dev = _device(fn, stream)
    i32, f32, bf = torch.int32, torch.float32, torch.bfloat16
    T, H, I, S = shape.T, shape.H, shape.I, shape.S
    if A13 is None or A13.dim() != 3:
        raise MoeError(f"{fn}: A13 must be [n_adapters, rank, H]", MOE_ERR_ARG)
    n, r = A13.shape[0], A13.shape[1]
    w, nw = _ws(fn, ws, dev)
    _check(fn, lib().moe_shared_ffn_adapted(
        ctypes.byref(shape), n, r, _arg(fn, "x", x, bf, T * H, dev), _arg(fn, "Wsh13", Wsh13, bf, S * 2 * I * H, dev),
        _arg(fn, "Wsh2", Wsh2, bf, S * H * I, dev), _arg(fn, "A13", A13, bf, n * r * H, dev),
        _arg(fn, "B13", B13, bf, n * S * 2 * I * r, dev), _arg(fn, "A2", A2, bf, n * r * S * I, dev),
        _arg(fn, "B2", B2, bf, n * H * r, dev), _arg(fn, "scale", scale, f32, n, dev),
        _arg(fn, "adapter_id", adapter_id, i32, T, dev), _arg(fn, "y_shared", y_shared, bf, T * H, dev),
        _arg(fn, "dev_status", dev_status, i32, 1, dev), w, nw, _stream(stream)))


def make_grouped_shape(P, K, M, E) -> MoeGroupedShape:
    return MoeGroupedShape(int(P), int(K), int(M), int(E), 0)


def moe_grouped_gemm(gshape, x, offsets, W, y, dev_status, stream=None):
    """y[p] = x[p] W_e^T for the rows p = offsets[e] .. offsets[e+1]-1 of each group e.  x [P,K], W [E,M,K], y [P,M] bf16;
    offsets int32 [E+1].  Rows outside every segment stay as they were."""
    fn = "moe_grouped_gemm"
    dev = _device(fn, stream)
    i32, bf, P, K, M, E = torch.int32, torch.bfloat16, gshape.P, gshape.K, gshape.M, gshape.E
    _check(fn, lib().moe_grouped_gemm(
        ctypes.byref(gshape), _arg(fn, "x", x, bf, P * K, dev), _arg(fn, "offsets", offsets, i32, E + 1, dev),
        _arg(fn, "W", W, bf, E * M * K, dev), _arg(fn, "y", y, bf, P * M, dev), _arg(fn, "dev_status", dev_status, i32, 1, dev),
        _handle(stream, dev)))


def moe_grouped_gemm_dx(gshape, dy, offsets, W, dx, dev_status, stream=None):
    """dx[p] = dy[p] W_e: the gradient of moe_grouped_gemm's rows.  dy [P,M], dx [P,K] bf16."""
    fn = "moe_grouped_gemm_dx"
    dev = _device(fn, stream)
    i32, bf, P, K, M, E = torch.int32, torch.bfloat16, gshape.P, gshape.K, gshape.M, gshape.E
    _check(fn, lib().moe_grouped_gemm_dx(
        ctypes.byref(gshape), _arg(fn, "dy", dy, bf, P * M, dev), _arg(fn, "offsets", offsets, i32, E + 1, dev),
        _arg(fn, "W", W, bf, E * M * K, dev), _arg(fn, "dx", dx, bf, P * K, dev), _arg(fn, "dev_status", dev_status, i32, 1, dev),
        _handle(stream, dev)))


def moe_grouped_gemm_dw(gshape, dy, x, offsets, dW, dev_status, add=False, stream=None):
    """dW_e = sum over the group's rows of dy[p]^T x[p]: the gradient of moe_grouped_gemm's weights, [E,M,K] bf16 or fp32.
    add: the sums are added to what dW holds (fp32 only)."""
    fn = "moe_grouped_gemm_dw"
    dev = _device(fn, stream)
    i32, bf, P, K, M, E = torch.int32, torch.bfloat16, gshape.P, gshape.K, gshape.M, gshape.E
    wide = dW is not None and dW.dtype is torch.float32
    s = MoeGroupedShape(P, K, M, E, gshape.flags | (MOE_GROUPED_DW_FP32 if wide else 0) | (MOE_GROUPED_DW_ADD if add else 0))
    _check(fn, lib().moe_grouped_gemm_dw(
        ctypes.byref(s), _arg(fn, "dy", dy, bf, P * M, dev), _arg(fn, "x", x, bf, P * K, dev),
        _arg(fn, "offsets", offsets, i32, E + 1, dev), _arg(fn, "dW", dW, torch.float32 if wide else bf, E * M * K, dev),
        _arg(fn, "dev_status", dev_status, i32, 1, dev), _handle(stream, dev)))


def moe_ffn_backward_workspace_bytes(shape: MoeShape, budget: int) -> int:
    return int(lib().moe_ffn_backward_workspace_bytes(ctypes.byref(shape), int(budget)))


def new_ffn_backward_workspace(shape: MoeShape, budget: int, device="cuda") -> torch.Tensor:
    n = moe_ffn_backward_workspace_bytes(shape, budget)
    if n == 0:
        raise MoeError("moe_ffn_backward_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_grouped_ffn_backward(shape, x_or_xperm, perm_token, expert_offsets, budget, W13, W2, d_y_perm, dx_perm, dW13, dW2,
                             dev_status, ws, stream=None):
    """Backward pass of moe_grouped_ffn: from the gradients of the experts' rows to those of the tokens' rows (dx_perm, in list
    order) and of both weights, all bf16; outputs that are None are not computed.  perm_token None: x_or_xperm is x_perm
    [budget,H]; else it is x [T,H] and row p is x[perm_token[p]]."""
    fn = "moe_grouped_ffn_backward"
    dev, budget = _device(fn, stream), int(budget)
    i32, bf, T, H, N, I = torch.int32, torch.bfloat16, shape.T, shape.H, shape.N, shape.I
    w, nw = _ws(fn, ws, dev)
    _check(fn, lib().moe_grouped_ffn_backward(
        ctypes.byref(shape), _arg(fn, "x_or_xperm", x_or_xperm, bf, (budget if perm_token is None else T) * H, dev, budget == 0),
        _arg(fn, "perm_token", perm_token, i32, budget, dev, True), _arg(fn, "expert_offsets", expert_offsets, i32, N + 1, dev), budget,
        _arg(fn, "W13", W13, bf, N * 2 * I * H, dev), _arg(fn, "W2", W2, bf, N * H * I, dev),
        _arg(fn, "d_y_perm", d_y_perm, bf, budget * H, dev, budget == 0), _arg(fn, "dx_perm", dx_perm, bf, budget * H, dev, True),
        _arg(fn, "dW13", dW13, bf, N * 2 * I * H, dev, True), _arg(fn, "dW2", dW2, bf, N * H * I, dev, True),
        _arg(fn, "dev_status", dev_status, i32, 1, dev), w, nw, _handle(stream, dev)))


def moe_shared_ffn_backward_workspace_bytes(shape: MoeShape) -> int:
    return int(lib().moe_shared_ffn_backward_workspace_bytes(ctypes.byref(shape)))


def new_shared_ffn_backward_workspace(shape: MoeShape, device="cuda") -> torch.Tensor:
    n = moe_shared_ffn_backward_workspace_bytes(shape)
    if n == 0:
        raise MoeError("moe_shared_ffn_backward_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_shared_ffn_backward(shape, x, Wsh13, Wsh2, d_y_shared, dx, dWsh13, dWsh2, dev_status, ws, stream=None):
    """Backward pass of moe_shared_ffn: from the gradient of the layer's output (weight one for every token) to those of the tokens and
    of both weights, all bf16; outputs that are None are not computed."""
    fn = "moe_shared_ffn_backward"
    dev = _device(fn, stream)
    i32, bf, T, H, I, S = torch.int32, torch.bfloat16, shape.T, shape.H, shape.I, shape.S
    w, nw = _ws(fn, ws, dev)
    _check(fn, lib().moe_shared_ffn_backward(
        ctypes.byref(shape), _arg(fn, "x", x, bf, T * H, dev), _arg(fn, "Wsh13", Wsh13, bf, S * 2 * I * H, dev),
        _arg(fn, "Wsh2", Wsh2, bf, S * H * I, dev), _arg(fn, "d_y_shared", d_y_shared, bf, T * H, dev),
        _arg(fn, "dx", dx, bf, T * H, dev, True), _arg(fn, "dWsh13", dWsh13, bf, S * 2 * I * H, dev, True),
        _arg(fn, "dWsh2", dWsh2, bf, S * H * I, dev, True), _arg(fn, "dev_status", dev_status, i32, 1, dev), w, nw, _handle(stream, dev)))


def make_norm_shape(T, H, gate_cols=0, eps=1e-6, y_as_is=False) -> MoeNormShape:
    return MoeNormShape(int(T), int(H), int(gate_cols), float(eps), MOE_NORM_Y_AS_IS if y_as_is else 0)


def moe_block_norm(nshape, r, y, w_post, gate, scale, w_pre, r_out, n_out, stream=None):
    """r_out = r + scale sigmoid(gate) w_post norm(y);  n_out = w_pre norm(r_out): the step between two blocks of a residual stack.
    r, y, r_out, n_out [T,H] and gate [T,gate_cols] bf16; w_post, w_pre [H] and scale [1] fp32.  None: gate, scale and gains of
    one; n_out not computed; y and r_out both None: n_out = w_pre norm(r)."""
    fn = "moe_block_norm"
    dev = _device(fn, stream)
    f32, bf, T, H, G = torch.float32, torch.bfloat16, nshape.T, nshape.H, nshape.gate_cols
    _check(fn, lib().moe_block_norm(
        ctypes.byref(nshape), _arg(fn, "r", r, bf, T * H, dev), _arg(fn, "y", y, bf, T * H, dev, True),
        _arg(fn, "w_post", w_post, f32, H, dev, True), _arg(fn, "gate", gate, bf, T * G, dev, True),
        _arg(fn, "scale", scale, f32, 1, dev, True), _arg(fn, "w_pre", w_pre, f32, H, dev, True),
        _arg(fn, "r_out", r_out, bf, T * H, dev, True), _arg(fn, "n_out", n_out, bf, T * H, dev, True), _handle(stream, dev)))


def moe_norm_workspace_bytes(nshape: MoeNormShape) -> int:
    return int(lib().moe_norm_workspace_bytes(ctypes.byref(nshape)))


def new_norm_workspace(nshape: MoeNormShape, device="cuda") -> torch.Tensor:
    n = moe_norm_workspace_bytes(nshape)
    if n == 0:
        raise MoeError("moe_norm_workspace_bytes", MOE_ERR_ARG)
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_block_norm_backward(nshape, r_out, y, w_post, gate, scale, w_pre, d_n, d_r_out, d_r, d_y, d_gate, dw_post, dw_pre, d_scale, ws=None,
                            stream=None):
    """Backward pass of moe_block_norm from the gradients of n_out (d_n) and r_out (d_r_out), either of which may be None.  Outputs
    that are None are not computed; ws is needed for dw_post, dw_pre and d_scale."""
    fn = "moe_block_norm_backward"
    dev = _device(fn, stream)
    f32, bf, T, H, G = torch.float32, torch.bfloat16, nshape.T, nshape.H, nshape.gate_cols
    w, nw = (None, 0) if ws is None else _ws(fn, ws, dev)
    _check(fn, lib().moe_block_norm_backward(
        ctypes.byref(nshape), _arg(fn, "r_out", r_out, bf, T * H, dev, d_n is None), _arg(fn, "y", y, bf, T * H, dev, True),
        _arg(fn, "w_post", w_post, f32, H, dev, True), _arg(fn, "gate", gate, bf, T * G, dev, True),
        _arg(fn, "scale", scale, f32, 1, dev, True), _arg(fn, "w_pre", w_pre, f32, H, dev, True), _arg(fn, "d_n", d_n, bf, T * H, dev, True),
        _arg(fn, "d_r_out", d_r_out, bf, T * H, dev, True), _arg(fn, "d_r", d_r, bf, T * H, dev, True),
        _arg(fn, "d_y", d_y, bf, T * H, dev, True), _arg(fn, "d_gate", d_gate, bf, T * G, dev, True),
        _arg(fn, "dw_post", dw_post, f32, H, dev, True), _arg(fn, "dw_pre", dw_pre, f32, H, dev, True),
        _arg(fn, "d_scale", d_scale, f32, 1, dev, True), w, nw, _handle(stream, dev)))


class AdamwTensors:
    """An optimizer's list for moe_adamw_step: the C entries and the tensors behind them, which it keeps alive."""

    def __init__(self, entries, tensors, device, sizes, states8):
        self.entries, self.tensors, self.device, self.sizes, self.states8 = entries, tensors, device, sizes, states8

    def __len__(self):
        return len(self.sizes)


def make_adamw_tensors(items) -> AdamwTensors:
    """items: one dict a tensor with param (fp32 or bf16), grad (fp32 or bf16), m and v (both fp32, or both uint8 with m_scale and
    v_scale fp32 [ceil(n / 256)]), and optionally copy (bf16) and weight_decay (0).  Made once; the tensors' contents may change
    from step to step, their memory may not."""
    fn = "make_adamw_tensors"
    items = list(items)
    if not items or not all(isinstance(it, dict) for it in items):
        raise MoeError(f"{fn}: items must be dicts, one at least", MOE_ERR_ARG)
    first = items[0].get("param")
    dev = first.get_device() if first is not None else -1
    if dev < 0:
        raise MoeError(f"{fn}: param must be a tensor on a CUDA device", MOE_ERR_ARG)
    f32, bf, u8 = torch.float32, torch.bfloat16, torch.uint8
    entries, kept, sizes, eight, written = (MoeAdamwTensor * len(items))(), [], [], [], []
    for k, it in enumerate(items):
        p, g, m = it.get("param"), it.get("grad"), it.get("m")
        if p is None or g is None or m is None or p.dtype not in (f32, bf) or g.dtype not in (f32, bf) or m.dtype not in (f32, u8):
            raise MoeError(f"{fn}: entry {k}: param and grad must be fp32 or bf16, m fp32 or uint8", MOE_ERR_ARG)
        n, s8 = p.numel(), m.dtype is u8
        blocks = -(-n // ADAMW_BLOCK)
        e = entries[k]
        e.param = _arg(fn, f"param of entry {k}", p, p.dtype, n, dev)
        e.grad = _arg(fn, f"grad of entry {k}", g, g.dtype, n, dev)
        e.m = _arg(fn, f"m of entry {k}", m, m.dtype, n, dev)
        e.v = _arg(fn, f"v of entry {k}", it.get("v"), m.dtype, n, dev)
        e.copy = _arg(fn, f"copy of entry {k}", it.get("copy"), bf, n, dev, True)
        if s8:
            e.m_scale = _arg(fn, f"m_scale of entry {k}", it.get("m_scale"), f32, blocks, dev)
            e.v_scale = _arg(fn, f"v_scale of entry {k}", it.get("v_scale"), f32, blocks, dev)
        e.n, e.weight_decay = n, float(it.get("weight_decay", 0.0))
        e.flags = ((MOE_ADAMW_PARAM_BF16 if p.dtype is bf else 0) | (MOE_ADAMW_GRAD_BF16 if g.dtype is bf else 0)
                   | (MOE_ADAMW_STATE8 if s8 else 0))
        names = ("param", "m", "v", "copy") + (("m_scale", "v_scale") if s8 else ())
        for name in names + ("grad",):
            t = it.get(name)
            if t is not None and n > 0:
                written.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), name != "grad", k, name))
        kept.append(dict(it))
        sizes.append(n)
        eight.append(s8)
    written.sort()
    reach = None                                # the entry that reaches furthest so far
    reach_written = None                        # the same among those that are written
    for w in written:
        for r in ((reach if w[2] else None), reach_written):
            if r is not None and w[0] < r[1]:
                raise MoeError(f"{fn}: {w[4]} of entry {w[3]} and {r[4]} of entry {r[3]} share memory", MOE_ERR_ARG)
        reach = w if reach is None or w[1] > reach[1] else reach
        if w[2]:
            reach_written = w if reach_written is None or w[1] > reach_written[1] else reach_written
    return AdamwTensors(entries, kept, dev, sizes, eight)


def _adamw_list(fn: str, tensors: AdamwTensors, stream) -> int:
    dev = _device(fn, stream)
    if not isinstance(tensors, AdamwTensors) or tensors.device != dev:
        raise MoeError(f"{fn}: tensors must come from make_adamw_tensors, on cuda:{dev}", MOE_ERR_ARG)
    return dev


def moe_adamw_step(tensors, beta1, beta2, eps, hyper, dev_status, stream=None):
    """One AdamW step over the list.  hyper fp32 [4] on the device: learning rate, 1 - beta1^t, 1 - beta2^t, factor of the
    gradients."""
    fn = "moe_adamw_step"
    dev = _adamw_list(fn, tensors, stream)
    _check(fn, lib().moe_adamw_step(tensors.entries, len(tensors), beta1, beta2, eps, _arg(fn, "hyper", hyper, torch.float32, 4, dev),
                                    _arg(fn, "dev_status", dev_status, torch.int32, 1, dev), _handle(stream, dev)))


def _state_values(fn: str, tensors: AdamwTensors, values, name: str, dev: int):
    if len(values) != len(tensors):
        raise MoeError(f"{fn}: {name} must hold one tensor an entry", MOE_ERR_ARG)
    out = (ctypes.c_void_p * len(values))()
    for k, (t, n) in enumerate(zip(values, tensors.sizes)):
        out[k] = _arg(fn, f"{name}[{k}]", t, torch.float32, n, dev)
    return out


def moe_adamw_states_read(tensors, m32, v32, stream=None):
    """The 8-bit states of the list as fp32 values: m32, v32 lists of fp32 tensors, one an entry."""
    fn = "moe_adamw_states_read"
    dev = _adamw_list(fn, tensors, stream)
    m, v = _state_values(fn, tensors, m32, "m32", dev), _state_values(fn, tensors, v32, "v32", dev)
    if len({*m, *v}) != 2 * len(tensors):
        raise MoeError(f"{fn}: m32 and v32 hold the same memory twice", MOE_ERR_ARG)
    _check(fn, lib().moe_adamw_states_read(tensors.entries, len(tensors), m, v, _handle(stream, dev)))


def moe_adamw_states_write(tensors, m32, v32, dev_status, stream=None):
    """Sets the 8-bit states of the list from fp32 values."""
    fn = "moe_adamw_states_write"
    dev = _adamw_list(fn, tensors, stream)
    _check(fn, lib().moe_adamw_states_write(tensors.entries, len(tensors), _state_values(fn, tensors, m32, "m32", dev),
                                            _state_values(fn, tensors, v32, "v32", dev),
                                            _arg(fn, "dev_status", dev_status, torch.int32, 1, dev), _handle(stream, dev)))


def moe_rmsnorm(shape, x, out, stream=None):
    _check("moe_rmsnorm", lib().moe_rmsnorm(ctypes.byref(shape), _p(x), _p(out), _stream(stream)))


def moe_layer_intermediates(shape, budget, ws) -> Dict[str, torch.Tensor]:
    """Views (copies to fresh tensors) of the routing intermediates a forward call left in `ws`."""
    ptrs = [ctypes.c_void_p() for _ in range(7)]
    _check("moe_layer_intermediates",
           lib().moe_layer_intermediates(ctypes.byref(shape), int(budget), _p(ws), ws.numel(),
                                         *[ctypes.byref(p) for p in ptrs]))
    base = ws.data_ptr()
    T, K, N, H, B = shape.T, shape.K_orig, shape.N, shape.H, int(budget)

    def view(ptr, nbytes, dtype, dims):
        off = ptr.value - base
        return ws[off:off + nbytes].view(dtype).reshape(*dims).clone()
    return dict(
        topk_idx=view(ptrs[0], T * K * 4, torch.int32, (T, K)),
        topk_score=view(ptrs[1], T * K * 4, torch.float32, (T, K)),
        n_sel=view(ptrs[2], T * 4, torch.int32, (T,)),
        expert_offsets=view(ptrs[3], (N + 1) * 4, torch.int32, (N + 1,)),
        perm_token=view(ptrs[4], B * 4, torch.int32, (B,)),
        pair_pos=view(ptrs[5], T * K * 4, torch.int32, (T, K)),
        y_perm=view(ptrs[6], B * H * 2, torch.bfloat16, (B, H)),
    )


def moe_profile_enable(on: bool):
    _check("moe_profile_enable", lib().moe_profile_enable(int(bool(on))))


def moe_profile_read() -> Dict[str, float]:
    """Device milliseconds of the six stages of the last moe_layer_forward call."""
    buf = (ctypes.c_float * len(PROFILE_STAGES))()
    _check("moe_profile_read", lib().moe_profile_read(buf))
    return {k: float(buf[i]) for i, k in enumerate(PROFILE_STAGES)}
