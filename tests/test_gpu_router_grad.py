"""The balance loss and the router's gradients against the fp64 oracle.

Tolerances come from counting roundings (u = 2^-24 for fp32, 2^-8 for bf16) and are stated where they are used."""
import numpy as np
import pytest
import torch

from oracle import adapt_oracle as ado
from paper_2604_08133_b200 import binding as B
from paper_2604_08133_b200 import synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
UB = 2.0 ** -8
i32, f32, bf16 = torch.int32, torch.float32, torch.bfloat16


def _routing(T, N, K, seed):
    """Softmax rows, their sorted Top-K and kept counts in 0..K (all from the seed)."""
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn(T, N, generator=g)
    s = torch.softmax(logits, 1)
    top = torch.topk(s, K, dim=1)
    n_sel = torch.randint(0, K + 1, (T,), generator=g, dtype=i32)
    return g, s.contiguous(), top.indices.to(i32).contiguous(), top.values.contiguous(), n_sel


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _ni(t):
    return None if t is None else t.detach().cpu().numpy()


# T, N, K, offsets: one token, one sequence, ragged ones, sequences that end inside a warp's rows, at its border, over many
# CTAs, empty ones (first, middle, last), padding before and behind
SEQ_CASES = [
    (1, 8, 1, None), (1, 8, 2, [0, 1]), (1, 8, 2, [0, 0]), (5, 60, 4, [0, 2, 2, 5]), (31, 64, 6, None), (64, 64, 6, [0, 32, 64]),
    (257, 128, 8, [3, 40, 41, 41, 256]), (700, 12, 3, [0, 256, 512, 700]), (700, 36, 3, [0, 255, 513, 700]),
    (1000, 64, 6, [0, 999]), (3000, 64, 6, None), (3001, 100, 16, [7, 7, 300, 2900, 2900, 2999]),
    (2048, 64, 2, list(range(0, 2049, 1))), (4111, 16, 4, [0] * 40 + [4000] + [4100] * 50),
]


def _ids(c):
    return "T%d-N%d-K%d-%s" % (c[0], c[1], c[2], "all" if c[3] is None else "%dseq" % (len(c[3]) - 1))


def _balance(T, N, K, off, seed=1, n_sel=True, alpha=0.3, fill=-7.0):
    g, s, idx, _, n = _routing(T, N, K, seed)
    n = n if n_sel else None
    offs = None if off is None else torch.tensor(off, dtype=i32)
    b = 1 if off is None else len(off) - 1
    shape = B.make_shape(T, 64, N, 64, 0, K, 0)
    out = dict(counts=torch.full((b, N), int(fill), dtype=i32, device="cuda"), coef=torch.full((b, N), fill, device="cuda"),
               loss=torch.full((1,), fill, device="cuda"))
    st = torch.zeros(1, dtype=i32, device="cuda")
    ws = B.new_router_workspace(shape, b)
    ws.fill_(255)
    d = lambda t: None if t is None else t.cuda()
    B.moe_balance_loss(shape, d(s), d(idx), d(n), d(offs), alpha, out["counts"], out["coef"], out["loss"], st, ws)
    torch.cuda.synchronize()
    return s, idx, n, out, int(st.item())


def _check_balance(T, N, s, idx, n, off, alpha, out):
    counts, coef, loss = ado.balance_loss(_np(s), _ni(idx), _ni(n), off, alpha)
    assert np.array_equal(out["counts"].cpu().numpy(), counts)
    # coef: conversions of c and C, c/C, alpha N / n_seq (two roundings, alpha itself one), the product, the division
    assert np.all(np.abs(_np(out["coef"]) - coef) <= 8 * U * coef)
    # loss: positive terms; a column's sum passes 32 additions in a warp, 3 shuffles, 8 in a CTA and one per further
    # partial on its way; then N/32 products, 5 shuffles, and the sequences' terms
    adds = 32 + 8 + 8 + T // 32 + N // 32 + 10 + (1 if off is None else len(off))
    assert abs(float(out["loss"]) - loss) <= (adds + 8) * U * loss


@pytest.mark.parametrize("case", SEQ_CASES, ids=_ids)
@pytest.mark.parametrize("with_n_sel", [True, False])
def test_balance_loss(case, with_n_sel):
    T, N, K, off = case
    s, idx, n, out, st = _balance(T, N, K, off, n_sel=with_n_sel)
    assert st == 0
    _check_balance(T, N, s, idx, n, off, np.float32(0.3).astype(np.float64), out)


@pytest.mark.parametrize("T,n_seq", [(1, 3000), (200, 64), (200, 65), (256, 700), (257, 5000)])
def test_balance_loss_of_many_sequences_and_few_rows(T, n_seq):
    """Most sequences empty; a long one, and short ones at both ends."""
    off = [0] * (n_seq // 2) + [T * 3 // 4] * (n_seq - n_seq // 2) + [T]
    s, idx, n, out, st = _balance(T, 64, 6, off)
    assert st == 0
    _check_balance(T, 64, s, idx, n, off, np.float32(0.3).astype(np.float64), out)


def test_balance_loss_of_a_long_packed_batch():
    """65 521 rows: hundreds of CTAs, the partials of long sequences joined; vectorised fp64 reference."""
    T, N, K = 65521, 64, 6
    off = [0, 5, 40000, 40000, 40257, 64718]
    s, idx, n, out, st = _balance(T, N, K, off)
    assert st == 0
    _check_balance(T, N, s, idx, n, off, np.float32(0.3).astype(np.float64), out)


def test_balance_loss_is_the_same_every_time_and_leaves_no_trace_in_the_workspace():
    T, N, K, off = 3001, 64, 6, [0, 17, 2900, 2999]
    ref = None
    for seed_ws in range(3):
        _, _, _, out, _ = _balance(T, N, K, off, fill=float(seed_ws))
        bits = [out["counts"].clone(), out["coef"].view(i32).clone(), out["loss"].view(i32).clone()]
        if ref is not None:
            assert all(torch.equal(a, b) for a, b in zip(ref, bits))
        ref = bits


def test_balance_loss_reports_bad_inputs_and_stays_in_bounds():
    T, N, K = 400, 64, 6
    shape = B.make_shape(T, 64, N, 64, 0, K, 0)
    _, s, idx, _, n = _routing(T, N, K, 2)
    ws = B.new_router_workspace(shape, 3)

    def status(s=s, idx=idx, n=n, off=(0, 100, 300, 399)):
        st = torch.zeros(1, dtype=i32, device="cuda")
        c, k, l = torch.zeros(3, N, dtype=i32, device="cuda"), torch.zeros(3, N, device="cuda"), torch.zeros(1, device="cuda")
        B.moe_balance_loss(shape, s.cuda(), idx.cuda(), n.cuda(), torch.tensor(off, dtype=i32).cuda(), 1.0, c, k, l, st, ws)
        torch.cuda.synchronize()
        return int(st.item()), c, k, l

    assert status()[0] == 0
    for bad in (float("nan"), float("inf"), -0.25):
        t = s.clone()
        t[150, 7] = bad
        assert status(s=t)[0] == 1 << B.MOE_ERR_NONFINITE
        t = s.clone()
        t[399, 7] = bad                                     # a row of padding: not looked at
        st, c, k, l = status(s=t)
        assert st == 0 and torch.isfinite(l).all()
    for bad in (-1, N, 2 ** 31 - 1):
        t = idx.clone()
        t[120, 0] = bad
        m = n.clone()
        m[120] = 3
        assert status(idx=t, n=m)[0] == 1 << B.MOE_ERR_ARG
        m[120] = 0                                          # the column is not kept
        assert status(idx=t, n=m)[0] == 0
    for off in ((0, 300, 100, 399), (-5, 100, 300, 399), (0, 100, 300, 401), (0, 2 ** 31 - 1, 300, 400)):
        assert status(off=off)[0] & (1 << B.MOE_ERR_ARG)
    t = n.clone()
    t[10], t[20] = -3, 99                                   # clamped to [0, K]
    st, c, _, _ = status(n=t)
    want = ado.balance_loss(_np(s), _ni(idx), _ni(t), [0, 100, 300, 399], 1.0)[0]
    assert st == 0 and np.array_equal(c.cpu().numpy(), want)


# ------------------------------------------------------------------------------------------------ gate backward
def _gate_case(T, H, N, K, off, seed, use=("top", "coef"), want=("d_logits", "dx", "dW", "db"), n_sel=True, poison=False):
    g, s, idx, _, n = _routing(T, N, K, seed)
    n = n if n_sel else None
    b = 1 if off is None else len(off) - 1
    x = synth.normal_bf16((T, H), 1.0, seed + 100)
    W = synth.normal_bf16((H, N), 0.02, seed + 200)
    d_top = torch.randn(T, K, generator=g) * 0.1 if "top" in use else None
    coef = torch.rand(b, N, generator=g) * 0.05 if "coef" in use else None
    offs = None if off is None else torch.tensor(off, dtype=i32)
    if poison:     # what must not be read: columns that are not kept, rows of padding
        if d_top is not None and n is not None:
            d_top = torch.where(torch.arange(K)[None, :] < n[:, None], d_top, float("nan"))
        if off is not None:
            inside = torch.zeros(T, dtype=torch.bool)
            inside[off[0]:off[-1]] = True
            x, s = x.clone(), s.clone()
            x[~inside] = float("nan")
            s[~inside] = float("inf")
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    out = dict(d_logits=torch.full((T, N), -7.0, device="cuda"), dx=torch.full((T, H), -7.0, dtype=bf16, device="cuda"),
               dW=torch.full((H, N), -7.0, device="cuda"), db=torch.full((N,), -7.0, device="cuda"))
    out = {k: (v if k in want else None) for k, v in out.items()}
    st = torch.zeros(1, dtype=i32, device="cuda")
    ws = B.new_router_workspace(shape, b)
    ws.fill_(255)
    d = lambda t: None if t is None else t.cuda()
    B.moe_gate_backward(shape, d(x) if "dW" in want else None, d(W) if "dx" in want else None, d(s),
                        d(idx) if "top" in use else None, d(n), d(d_top), d(coef), d(offs), out["d_logits"], out["dx"],
                        out["dW"], out["db"], st, ws)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    _check_gate(T, H, N, K, off, x, W, s, idx, n, d_top, coef, out)
    return out


def _check_gate(T, H, N, K, off, x, W, s, idx, n, d_top, coef, out):
    inside = np.zeros(T, bool)
    for lo, hi in ado.sequences(off, T):
        inside[lo:hi] = True
    s64 = np.where(inside[:, None], _np(s), 0.0)
    x64 = np.where(inside[:, None], _np(x), 0.0)
    d, dx, dW, db = ado.gate_backward(x64, _np(W), s64, _ni(idx), _ni(n), _np(d_top), _np(coef), off)
    # d_logits = s (g - D): g takes up to K additions, D = sum s g is a chain of 4 FMAs and 5 shuffles, then the
    # difference and the product round once each
    _, g_abs = ado.score_gradient(T, N, _ni(idx), _ni(n), _np(d_top), _np(coef), off)
    D_abs = (s64 * g_abs).sum(1, keepdims=True)
    e_d = U * s64 * ((K + 2) * g_abs + (K + 12) * D_abs)
    if out["d_logits"] is not None:
        assert np.all(np.abs(_np(out["d_logits"]) - d) <= e_d), "d_logits"
    # two bf16 terms stand for d_logits within 2^-16 of it; products are exact in fp32, sums of n terms add n u
    e_two = UB * UB * np.abs(d) + e_d
    if out["dx"] is not None:
        terms = np.abs(d) @ np.abs(_np(W)).T
        tol = UB * np.abs(dx) + (1 + UB) * (e_two @ np.abs(_np(W)).T + 2 * N * U * terms)
        assert np.all(np.abs(_np(out["dx"]) - dx) <= tol), "dx"
    if out["dW"] is not None:
        terms = np.abs(x64).T @ np.abs(d)
        tol = np.abs(x64).T @ e_two + 2 * (T + 64) * U * terms
        assert np.all(np.abs(_np(out["dW"]) - dW) <= tol), "dW"
    if out["db"] is not None:
        assert np.all(np.abs(_np(out["db"]) - db) <= e_d.sum(0) + (T + 64) * U * np.abs(d).sum(0)), "db"


GATE_CASES = [(1, 64, 8, 1, None), (3, 128, 12, 2, [0, 2, 3]), (64, 256, 64, 6, None), (65, 320, 60, 4, [0, 30, 30, 65]),
              (129, 192, 128, 8, [5, 60, 120]), (300, 64, 36, 16, [0, 1, 2, 290]), (515, 512, 64, 6, [0, 128, 256, 515]),
              (1100, 2048, 8, 2, None), (2500, 576, 100, 5, [0, 1000, 2499]), (200, 64, 68, 3, [100, 100, 101])]


@pytest.mark.parametrize("case", GATE_CASES, ids=lambda c: "T%d-H%d-N%d-K%d-%s" % (*c[:4], "all" if c[4] is None else "seq"))
@pytest.mark.parametrize("use", [("top", "coef"), ("top",), ("coef",)], ids="+".join)
def test_gate_backward(case, use):
    _gate_case(*case, seed=7, use=use, poison=True)


@pytest.mark.parametrize("want", [("d_logits",), ("dx",), ("dW",), ("db",), ("dx", "db"), ("dW", "d_logits"), ("dx", "dW")],
                         ids="+".join)
@pytest.mark.parametrize("case", [(70, 128, 60, 4, [0, 40, 66]), (1300, 256, 64, 6, None)], ids=["odd", "long"])
def test_gate_backward_of_each_output_alone(case, want):
    _gate_case(*case, seed=9, want=want, n_sel=False)


def test_gate_backward_gives_padding_no_gradient_whatever_the_weights_hold():
    T, H, N, K = 300, 128, 64, 6
    g, s, idx, _, n = _routing(T, N, K, 5)
    W = torch.randn(H, N, generator=g).bfloat16()
    W[3, 4], W[100, 7] = float("inf"), float("nan")
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    off = torch.tensor([20, 140, 290], dtype=i32).cuda()
    dx = torch.full((T, H), 9.0, dtype=bf16, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    B.moe_gate_backward(shape, None, W.cuda(), s.cuda(), idx.cuda(), n.cuda(), torch.randn(T, K, generator=g).cuda(), None, off,
                        None, dx, None, None, st, B.new_router_workspace(shape, 2))
    torch.cuda.synchronize()
    assert st.item() == 0
    assert torch.all(dx[:20] == 0) and torch.all(dx[290:] == 0)
    rows = dx[20:290]
    assert not torch.isfinite(rows[:, [3, 100]]).any()
    keep = [h for h in range(H) if h not in (3, 100)]
    assert torch.isfinite(rows[:, keep]).all()


@pytest.mark.parametrize("N", [8, 32, 60, 128])
def test_gate_backward_of_an_overflowing_d_logits_is_infinite_not_nan(N):
    """g up to 3e38 in both directions: g - sum s g passes fp32's range, d_logits of one expert is infinite, and so are
    the sums that it enters; its other terms add nothing."""
    T, H = 70, 128
    g = torch.Generator().manual_seed(2)
    s = torch.softmax(torch.randn(T, N, generator=g), 1)
    s[11] = 0.0
    s[11, 0], s[11, 1] = 0.125, 0.875
    x = torch.rand(T, H, generator=g).add(0.5).bfloat16()
    W = torch.randn(H, N, generator=g).bfloat16()
    W[:, 0] = torch.where(torch.arange(H) % 2 == 0, 1.0, -2.0)
    off = torch.tensor([0, 11, 12, T], dtype=i32)
    coef = torch.rand(3, N, generator=g) * 0.05
    coef[1] = 0.0
    coef[1, 0], coef[1, 1] = 3e38, -3e38
    shape = B.make_shape(T, H, N, 64, 0, 2, 0)
    out = dict(d_logits=torch.zeros(T, N, device="cuda"), dx=torch.zeros(T, H, dtype=bf16, device="cuda"),
               dW=torch.zeros(H, N, device="cuda"), db=torch.zeros(N, device="cuda"))
    st = torch.zeros(1, dtype=i32, device="cuda")
    B.moe_gate_backward(shape, x.cuda(), W.cuda(), s.cuda(), None, None, None, coef.cuda(), off.cuda(), out["d_logits"], out["dx"],
                        out["dW"], out["db"], st, B.new_router_workspace(shape, 3))
    torch.cuda.synchronize()
    d, dx, dW, db = (out[k].float().cpu() for k in ("d_logits", "dx", "dW", "db"))
    assert d[11, 0] == float("inf") and torch.isfinite(d[11, 1:]).all() and db[0] == float("inf")
    assert torch.all(dx[11] == torch.where(W[:, 0] > 0, float("inf"), -float("inf")))
    assert torch.all(dW[:, 0] == float("inf")) and torch.isfinite(dW[:, 1:]).all()
    rest = torch.arange(T) != 11
    assert torch.isfinite(dx[rest]).all()


def test_gate_backward_with_no_rows_at_all():
    """Every sequence empty: all gradients are zero, whatever the inputs hold."""
    out = _gate_case(150, 128, 64, 6, [20, 20, 20], seed=4, poison=True)
    assert all(not v.float().any() for v in out.values())


def test_gate_backward_counts_an_expert_named_twice_twice():
    T, N, K = 33, 16, 4
    _, s, idx, _, n = _routing(T, N, K, 6)
    idx[:, 2] = idx[:, 0]
    g = torch.Generator().manual_seed(1)
    d_top = torch.randn(T, K, generator=g)
    shape = B.make_shape(T, 64, N, 64, 0, K, 0)
    out, st = torch.empty(T, N, device="cuda"), torch.zeros(1, dtype=i32, device="cuda")
    B.moe_gate_backward(shape, None, None, s.cuda(), idx.cuda(), None, d_top.cuda(), None, None, out, None, None, None, st,
                        B.new_router_workspace(shape))
    _check_gate(T, 64, N, K, None, torch.zeros(T, 64), torch.zeros(64, N), s, idx, None, d_top, None,
                dict(d_logits=out, dx=None, dW=None, db=None))
    assert int(st.item()) == 0
    idx[5, 1] = N                                             # reported, skipped
    B.moe_gate_backward(shape, None, None, s.cuda(), idx.cuda(), None, d_top.cuda(), None, None, out, None, None, None, st,
                        B.new_router_workspace(shape))
    assert int(st.item()) == 1 << B.MOE_ERR_ARG and torch.isfinite(out).all()


@pytest.mark.parametrize("N,K", [(8, 2), (16, 4), (32, 5), (64, 6), (128, 16)])
@pytest.mark.parametrize("bad", [-1, -2, "N", 2 ** 31 - 1, -2 ** 31])
def test_gate_backward_reports_every_id_outside_the_experts(N, K, bad):
    """A kept pair of any id outside [0, N) is skipped and reported; a column that is not kept, or a row of padding, may
    hold anything."""
    T, bad = 70, N if bad == "N" else bad
    _, s, idx, _, n = _routing(T, N, K, 6)
    off = [3, 30, 66]
    d_top = torch.randn(T, K, generator=torch.Generator().manual_seed(1))
    shape = B.make_shape(T, 64, N, 64, 0, K, 0)
    ws, offs = B.new_router_workspace(shape, 2), torch.tensor(off, dtype=i32).cuda()

    def call(idx, n):
        out, st = torch.empty(T, N, device="cuda"), torch.zeros(1, dtype=i32, device="cuda")
        B.moe_gate_backward(shape, None, None, s.cuda(), idx.cuda(), n.cuda(), d_top.cuda(), None, offs, out, None, None, None, st, ws)
        return out, int(st.item())

    for col in {0, K - 1}:
        n[40] = col + 1
        t = idx.clone()
        t[40, col] = bad
        out, st = call(t, n)
        assert st == 1 << B.MOE_ERR_ARG
        zeroed = d_top.clone()                                # the pair adds nothing
        zeroed[40, col] = 0.0
        _check_gate(T, 64, N, K, off, torch.zeros(T, 64), torch.zeros(64, N), s, idx, n, zeroed, None,
                    dict(d_logits=out, dx=None, dW=None, db=None))
        m = n.clone()
        m[40] = col                                           # not kept
        assert call(t, m)[1] == 0
    t = idx.clone()
    t[1], t[68] = bad, bad                                    # padding
    assert call(t, n)[1] == 0


def test_gate_backward_is_the_same_every_time():
    a = _gate_case(1300, 256, 64, 6, [0, 700, 1250], seed=3)
    for _ in range(3):
        b = _gate_case(1300, 256, 64, 6, [0, 700, 1250], seed=3)
        assert all(torch.equal(a[k].view(torch.int16 if a[k].dtype is bf16 else i32),
                               b[k].view(torch.int16 if b[k].dtype is bf16 else i32)) for k in a)


# ------------------------------------------------------------------------------------------------ combine backward
@pytest.mark.parametrize("T,H,N,K,kept", [(1, 64, 8, 1, None), (1, 64, 8, 2, [0]), (7, 320, 8, 3, None), (64, 2048, 64, 6, None),
                                          (33, 4096, 60, 16, None), (300, 128, 16, 4, None)])
@pytest.mark.parametrize("with_rows", [True, False])
def test_combine_backward(T, H, N, K, kept, with_rows):
    g, _, idx, score, n = _routing(T, N, K, 13)
    if kept is not None:
        n = torch.tensor(kept, dtype=i32)
    budget = int(n.sum())
    room = min(budget + 2, T * K)                            # rows that no pair names stay as they were
    order = torch.randperm(room, generator=g)[:budget].to(i32)
    pos = torch.full((T, K), -1, dtype=i32)
    pos[torch.arange(K)[None, :] < n[:, None]] = order
    y = synth.normal_bf16((room, H), 0.5, 41)
    d_out = synth.normal_bf16((T, H), 1.0, 43)
    d_y = torch.full((room, H), -7.0, dtype=bf16, device="cuda") if with_rows else None
    d_s = torch.full((T, K), -7.0, device="cuda")
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    B.moe_combine_backward(shape, d_out.cuda(), y.cuda(), pos.cuda(), score.cuda() if with_rows else None, n.cuda(), room, d_s, d_y)
    torch.cuda.synchronize()
    want_s, want_y = ado.combine_backward(_np(d_out), _np(y), _ni(pos), _np(score), _ni(n), np.full((room, H), -7.0))
    bound = np.zeros((T, K))
    for t in range(T):
        for j in range(int(n[t])):
            bound[t, j] = (np.abs(_np(d_out[t])) * np.abs(_np(y[int(pos[t, j])]))).sum()
    # the dot product: at most H / 32 FMAs a lane (products exact), a few joins of partial sums
    assert np.all(np.abs(_np(d_s) - want_s) <= (H / 32 + 16) * U * bound)
    if with_rows:                                            # one fp32 product, one rounding to bf16
        assert np.all(np.abs(_np(d_y) - want_y) <= (UB + 2 * U) * np.abs(want_y))


def test_combine_backward_with_no_rows_at_all():
    shape = B.make_shape(9, 64, 8, 64, 0, 2, 0)
    d_s = torch.full((9, 2), -7.0, device="cuda")
    B.moe_combine_backward(shape, torch.ones(9, 64, dtype=bf16, device="cuda"), torch.zeros(0, 64, dtype=bf16, device="cuda"),
                           torch.zeros(9, 2, dtype=i32, device="cuda"), None, torch.ones(9, dtype=i32, device="cuda"), 0, d_s, None)
    torch.cuda.synchronize()
    assert not d_s.any()


def test_combine_backward_ignores_what_is_not_kept():
    """Positions and rows behind a token's kept columns are not used, and positions outside the list count as not kept."""
    T, H, K = 40, 128, 4
    g = torch.Generator().manual_seed(2)
    shape = B.make_shape(T, H, 8, 64, 0, K, 0)
    n = torch.randint(0, K + 1, (T,), generator=g, dtype=i32)
    pos = torch.arange(T * K, dtype=i32).view(T, K).clone()
    pos[3, 0], pos[4, 0] = 2 ** 31 - 1, -5
    n[3], n[4] = 2, 1
    y = synth.normal_bf16((T * K, H), 1.0, 3)
    y.view(T, K, H)[torch.arange(K)[None, :] >= n[:, None]] = float("nan")
    score = torch.rand(T, K, generator=g)
    d_out = synth.normal_bf16((T, H), 1.0, 4)
    d_s = torch.full((T, K), -7.0, device="cuda")
    d_y = torch.full((T * K, H), -7.0, dtype=bf16, device="cuda")
    B.moe_combine_backward(shape, d_out.cuda(), y.cuda(), pos.cuda(), score.cuda(), n.cuda(), T * K, d_s, d_y)
    torch.cuda.synchronize()
    kept = (torch.arange(K)[None, :] < n[:, None])
    kept[3, 0] = kept[4, 0] = False
    assert torch.isfinite(d_s).all() and not d_s.cpu()[~kept].any()
    assert (d_y.cpu().view(T, K, H)[~kept] == -7.0).all()
    want = _np(score[:, :, None] * d_out.float()[:, None, :])[kept.numpy()]
    assert np.all(np.abs(_np(d_y).reshape(T, K, H)[kept.numpy()] - want) <= (UB + 2 * U) * np.abs(want))


# ------------------------------------------------------------------------------------------------ together, graphs
def _router_step(dev_inputs, bufs, shape, budget, off):
    """What a router update does: gate, selection, routing lists; Eq. 2's gradient, the balance loss, the gate's gradient."""
    x, W, bias, y, d_out = dev_inputs
    b = bufs
    B.moe_gate(shape, x, W, bias, b["scores"], b["idx"], b["top"])
    B.moe_route(shape, b["idx"], b["top"], budget, b["n_sel"], b["offs"], b["tok"], b["wgt"], b["pos"], b["st"])
    B.moe_combine_backward(shape, d_out, y, b["pos"], None, b["n_sel"], budget, b["d_top"], None)
    B.moe_balance_loss(shape, b["scores"], b["idx"], b["n_sel"], off, 0.01, b["counts"], b["coef"], b["loss"], b["st"], b["ws"])
    B.moe_gate_backward(shape, x, W, b["scores"], b["idx"], b["n_sel"], b["d_top"], b["coef"], off, None, b["dx"], b["dW"], b["db"],
                        b["st"], b["ws"])


def _step_setup(T=600, H=256, N=64, K=6, seed=21):
    budget = 3 * T
    shape = B.make_shape(T, H, N, 64, 0, K, 1)
    c = lambda *s, dt=f32: torch.zeros(*s, dtype=dt, device="cuda")
    off = torch.tensor([0, 200, 550], dtype=i32, device="cuda")
    inputs = (synth.normal_bf16((T, H), 1.0, seed).cuda(), synth.normal_bf16((H, N), 0.05, seed + 1).cuda(),
              synth.normal_bf16((N,), 0.5, seed + 2).float().cuda(), synth.normal_bf16((budget, H), 0.5, seed + 3).cuda(),
              synth.normal_bf16((T, H), 1.0, seed + 4).cuda())
    bufs = dict(scores=c(T, N), idx=c(T, K, dt=i32), top=c(T, K), n_sel=c(T, dt=i32), offs=c(N + 1, dt=i32),
                tok=c(budget, dt=i32), wgt=c(budget), pos=c(T, K, dt=i32), d_top=c(T, K), counts=c(2, N, dt=i32), coef=c(2, N),
                loss=c(1), dx=c(T, H, dt=bf16), dW=c(H, N), db=c(N), st=c(1, dt=i32), ws=B.new_router_workspace(shape, 2))
    return shape, budget, off, inputs, bufs


def test_router_step_from_tokens_to_the_gates_gradient():
    shape, budget, off, inputs, b = _step_setup()
    _router_step(inputs, b, shape, budget, off)
    torch.cuda.synchronize()
    assert int(b["st"].item()) == 0
    T, H, N, K = shape.T, shape.H, shape.N, shape.K_orig
    offs = off.cpu().tolist()
    _check_balance(T, N, b["scores"], b["idx"], b["n_sel"], offs, float(np.float32(0.01)), b)
    want_s, _ = ado.combine_backward(_np(inputs[4]), _np(inputs[3]), _ni(b["pos"]), np.zeros((T, K)), _ni(b["n_sel"]),
                                     np.zeros((budget, H)))
    assert np.abs(_np(b["d_top"]) - want_s).max() <= (H / 32 + 16) * U * H * 36   # |d_out|, |y| < 6 standard deviations
    _check_gate(T, H, N, K, offs, inputs[0], inputs[1], b["scores"], b["idx"], b["n_sel"], b["d_top"], b["coef"],
                dict(d_logits=None, dx=b["dx"], dW=b["dW"], db=b["db"]))


def test_router_step_on_a_side_stream_and_replayed_from_a_graph():
    shape, budget, off, inputs, b = _step_setup()
    _router_step(inputs, b, shape, budget, off)
    torch.cuda.synchronize()
    keys = ("loss", "coef", "dW", "db", "dx")
    ref = {k: b[k].clone() for k in keys}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in keys:
            b[k].fill_(3)
        _router_step(inputs, b, shape, budget, off)
    side.synchronize()
    assert all(torch.equal(ref[k], b[k]) for k in keys)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _router_step(inputs, b, shape, budget, off)
    for _ in range(2):
        for k in keys:
            b[k].fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(ref[k], b[k]) for k in keys)
    inputs[0].neg_()                                          # other inputs in the same buffers: nothing was remembered
    graph.replay()
    torch.cuda.synchronize()
    again = {k: b[k].clone() for k in keys}
    _router_step(inputs, b, shape, budget, off)
    torch.cuda.synchronize()
    assert all(torch.equal(again[k], b[k]) for k in keys) and not torch.equal(again["dW"], ref["dW"])


# ------------------------------------------------------------------------------------------------ what the terms hold
@pytest.mark.parametrize("T", [1, 2])
@pytest.mark.parametrize("N", [8, 16, 60, 64, 100, 128])
def test_dW_holds_d_logits_to_24_bits(T, N):
    """Tokens of +-1: dW is d_logits itself, or the sum of two.  Two of its three bf16 terms would be off by up to 2^-18."""
    H, K = 128, 2
    g, s, idx, _, _ = _routing(T, N, K, N + T)
    coef = torch.randn(1, N, generator=g)
    x = torch.where(torch.rand(T, H, generator=g) < 0.5, -1.0, 1.0).bfloat16()
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    d, dW = torch.zeros(T, N, device="cuda"), torch.zeros(H, N, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    B.moe_gate_backward(shape, x.cuda(), None, s.cuda(), None, None, None, coef.cuda(), None, d, None, dW, None, st,
                        B.new_router_workspace(shape))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want, terms = _np(x).T @ _np(d), np.abs(_np(x)).T @ np.abs(_np(d))
    # against the d_logits that the call returned: 2^-24 of each, and 3 T additions of its terms (truncated: 2 U each)
    assert np.all(np.abs(_np(dW) - want) <= (2.0 ** -24 + 2 * 3 * T * U) * terms)


@pytest.mark.parametrize("T", [1, 70, 300])
@pytest.mark.parametrize("N", [8, 16, 60, 64, 100, 128])
def test_dx_holds_d_logits_to_16_bits(T, N):
    """A row of d_logits adds up to nothing, so with equal weights dx is what its terms leave: one bf16 term would leave
    2^-9 of them."""
    H, K = 128, 2
    g, s, idx, _, _ = _routing(T, N, K, N + T)
    coef = torch.randn(1, N, generator=g)
    W = (torch.randn(H, 1, generator=g) * torch.ones(1, N)).bfloat16()
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    d, dx = torch.zeros(T, N, device="cuda"), torch.zeros(T, H, dtype=bf16, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    B.moe_gate_backward(shape, None, W.cuda(), s.cuda(), None, None, None, coef.cuda(), None, d, dx, None, None, st,
                        B.new_router_workspace(shape))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want, terms = _np(d) @ _np(W).T, np.abs(_np(d)) @ np.abs(_np(W)).T
    e = (2.0 ** -16 + 2 * 2 * N * U) * terms
    assert np.all(np.abs(_np(dx) - want) <= e + UB * (np.abs(want) + e))
    assert np.abs(want).max() <= 2.0 ** -12 * terms.max()         # or the rounding of dx would hide the terms


# ------------------------------------------------------------------------------------------------ ends of the ranges
@pytest.mark.parametrize("case", [(700, 3200, 8, 2, [0, 300, 690]), (900, 6144, 12, 3, None), (300, 20480, 16, 2, [1, 299]),
                                  (300, 1216, 128, 16, None), (1500, 128, 32, 8, None)],
                         ids=lambda c: "T%d-H%d-N%d-K%d" % c[:4])
def test_gate_backward_with_clusters_of_every_size(case):
    """Slices of H that leave one, three, five and six CTAs a slice."""
    _gate_case(*case, seed=17, poison=True)


@pytest.mark.parametrize("T,n_seq", [(1, 3000), (257, 5000), (600, 700)])
def test_gate_backward_with_more_sequences_than_rows(T, n_seq):
    off = [0] * (n_seq // 2) + [T * 3 // 4] * (n_seq - n_seq // 2) + [T]
    _gate_case(T, 128, 64, 6, off, seed=18)


def _at_offset(t, elems):
    """The same tensor 16 bytes behind an aligned address."""
    raw = torch.empty(t.numel() + elems, dtype=t.dtype, device="cuda")
    out = raw[elems:].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("N", [8, 60, 128])
def test_sixteen_byte_alignment_is_enough(N):
    T, H, K = 333, 320, 2
    g, s, idx, top, n = _routing(T, N, K, 19)
    off = torch.tensor([2, 100, 330], dtype=i32).cuda()
    x, W, d_top = synth.normal_bf16((T, H), 1.0, 1), synth.normal_bf16((H, N), 0.02, 2), torch.randn(T, K, generator=g)
    budget = int(n.sum())
    pos = torch.full((T, K), -1, dtype=i32)
    pos[torch.arange(K)[None, :] < n[:, None]] = torch.randperm(budget, generator=g).to(i32)
    y, d_out = synth.normal_bf16((budget, H), 1.0, 3), synth.normal_bf16((T, H), 1.0, 4)
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    outs = []
    for shift in (0, 1):
        a = lambda t: _at_offset(t, shift * 16 // t.element_size())
        z = lambda *v, dt=f32: a(torch.full(v, -7, dtype=dt))
        ws = torch.full((B.moe_router_workspace_bytes(shape, 2) + 16,), 255, dtype=torch.uint8, device="cuda")[16 * shift:]
        st = torch.zeros(1, dtype=i32, device="cuda")
        o = dict(counts=z(2, N, dt=i32), coef=z(2, N), loss=torch.zeros(1, device="cuda"), d_logits=z(T, N), dx=z(T, H, dt=bf16),
                 dW=z(H, N), db=z(N), d_s=z(T, K), d_y=z(budget, H, dt=bf16))
        sc, ix = a(s), a(idx)
        B.moe_balance_loss(shape, sc, ix, n.cuda(), off, 0.5, o["counts"], o["coef"], o["loss"], st, ws)
        B.moe_gate_backward(shape, a(x), a(W), sc, ix, n.cuda(), a(d_top), o["coef"], off, o["d_logits"], o["dx"], o["dW"], o["db"], st, ws)
        B.moe_combine_backward(shape, a(d_out), a(y), a(pos), a(top), n.cuda(), budget, o["d_s"], o["d_y"])
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        outs.append({k: v.cpu() for k, v in o.items()})
    assert all(torch.equal(outs[0][k], outs[1][k]) for k in outs[0])


def _needs(gigabytes):
    if torch.cuda.mem_get_info()[0] < (gigabytes + 10) * 10 ** 9:
        pytest.skip(f"needs {gigabytes} GB")


def test_balance_loss_of_more_scores_than_32_bits_count():
    """2.2e9 scores: row offsets beyond 2^31 in both directions of use."""
    _needs(40)
    T, N, K = 17_000_000, 128, 1
    g = torch.Generator(device="cuda").manual_seed(1)
    off = [5, T // 2 + 77, T - 3]
    s = torch.rand(T, N, device="cuda", generator=g) * (2.0 / N)
    idx = torch.randint(0, N, (T, K), device="cuda", generator=g, dtype=i32)
    shape = B.make_shape(T, 64, N, 64, 0, K, 0)
    out = dict(counts=torch.zeros(2, N, dtype=i32, device="cuda"), coef=torch.zeros(2, N, device="cuda"), loss=torch.zeros(1, device="cuda"))
    st = torch.zeros(1, dtype=i32, device="cuda")
    offs, ws = torch.tensor(off, dtype=i32, device="cuda"), B.new_router_workspace(shape, 2)
    B.moe_balance_loss(shape, s, idx, None, offs, 0.5, out["counts"], out["coef"], out["loss"], st, ws)
    d = torch.empty(T, N, device="cuda")
    B.moe_gate_backward(shape, None, None, s, None, None, None, out["coef"], offs, d, None, None, None, st, ws)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    loss = 0.0
    for b in range(2):
        lo, hi = off[b], off[b + 1]
        c = torch.bincount(idx[lo:hi, 0].long(), minlength=N)
        assert torch.equal(c, out["counts"][b].long())
        coef = 0.5 / 2 * N * c.double() / (hi - lo) / (hi - lo)
        assert torch.all((out["coef"][b] - coef).abs() <= 8 * U * coef)
        total = torch.zeros(N, dtype=torch.float64, device="cuda")
        for r in range(lo, hi, 1 << 20):
            total += s[r:min(hi, r + (1 << 20))].double().sum(0)
        loss += float((coef * total).sum())
    # a column's sum passes 32 rows, 8 warps, then one partial of 256 rows after the other over two threads' groups
    assert abs(float(out["loss"]) - loss) <= (32 + 8 + T // 256 + 64) * U * loss
    rows = torch.tensor([5, 6, T // 2, T // 2 + 77, T - 5, T - 4], device="cuda")
    seq = (rows >= off[1]).long()
    p, k = s[rows].double(), out["coef"][seq].double()
    want = p * (k - (p * k).sum(1, keepdim=True))
    e = 14 * U * p * (k + (p * k).sum(1, keepdim=True))
    assert torch.all((d[rows] - want).abs() <= e)
    assert not d[:5].any() and not d[T - 3:].any()
    del s, d, idx
    torch.cuda.empty_cache()


def test_gate_and_combine_backward_of_more_elements_than_32_bits_count():
    """4.3e9 elements of x and dx, as many of y_perm and d_y_perm."""
    _needs(60)
    T, H, N, K = 530_000, 8192, 8, 1
    g = torch.Generator(device="cuda").manual_seed(2)
    s = torch.softmax(torch.randn(T, N, device="cuda", generator=g), 1)
    x = torch.empty(T, H, dtype=bf16, device="cuda").normal_(generator=g)
    W = (torch.randn(H, N, device="cuda", generator=g) * 0.02).to(bf16)
    coef = torch.rand(1, N, device="cuda", generator=g)
    shape = B.make_shape(T, H, N, 64, 0, K, 0)
    d, dx, dW = torch.empty(T, N, device="cuda"), torch.empty(T, H, dtype=bf16, device="cuda"), torch.empty(H, N, device="cuda")
    db, st = torch.empty(N, device="cuda"), torch.zeros(1, dtype=i32, device="cuda")
    B.moe_gate_backward(shape, x, W, s, None, None, None, coef, None, d, dx, dW, db, st, B.new_router_workspace(shape))
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    rows = torch.cat([torch.arange(0, T, 9973), torch.arange(T - 40, T)]).cuda()
    want, terms = d[rows].double() @ W.double().T, d[rows].double().abs() @ W.double().abs().T
    e = (UB * UB + 2 * 2 * N * U) * terms
    assert torch.all((dx[rows].double() - want).abs() <= e + UB * (want.abs() + e))
    acc, mag = torch.zeros(H, N, dtype=torch.float64, device="cuda"), torch.zeros(H, N, dtype=torch.float64, device="cuda")
    for r in range(0, T, 1 << 16):
        xr, dr = x[r:r + (1 << 16)].double(), d[r:r + (1 << 16)].double()
        acc += xr.T @ dr
        mag += xr.abs().T @ dr.abs()
    # flushed every four blocks of 128 rows: three terms of 512 rows in one accumulator, then one addition a flush and CTA
    assert torch.all((dW.double() - acc).abs() <= (2.0 ** -24 + (2 * 3 * 512 + T // 512 + 16) * U) * mag)
    assert torch.all((db.double() - d.double().sum(0)).abs() <= (T // 296 + 400) * U * d.double().abs().sum(0))
    # the same buffers as Eq. 2's: x is y_perm, dx its gradient, every position once, in reverse
    pos = torch.arange(T - 1, -1, -1, device="cuda", dtype=i32).view(T, 1)
    d_out, w = x.roll(1, 0), torch.rand(T, 1, device="cuda", generator=g)
    n, d_s = torch.ones(T, dtype=i32, device="cuda"), torch.empty(T, 1, device="cuda")
    B.moe_combine_backward(shape, d_out, x, pos, w, n, T, d_s, dx)
    torch.cuda.synchronize()
    t = rows
    a, y = d_out[t].double(), x[T - 1 - t].double()
    assert torch.all((d_s[t, 0].double() - (a * y).sum(1)).abs() <= (H / 32 + 16) * U * (a * y).abs().sum(1))
    want = w[t].double() * a
    assert torch.all((dx[T - 1 - t].double() - want).abs() <= (UB + 2 * U) * want.abs())
    del x, dx, d_out
    torch.cuda.empty_cache()


def test_router_steps_and_adapters_at_the_same_time():
    """Three streams: two router updates and adapted projections of few and of many tokens, a workspace each, overlapping
    as they like."""
    steps = [_step_setup(T=600, seed=21), _step_setup(T=1300, H=512, N=64, seed=51)]
    keys = ("loss", "coef", "dW", "db", "dx")
    adapters = []
    for T, K, M, n, r, seed in ((5, 64, 128, 3, 8, 1), (64, 512, 1032, 16, 16, 2), (700, 256, 1032, 16, 24, 3)):
        s = B.make_adapter_shape(T, K, M, n, r)
        ids = torch.randint(-1, n, (T,), generator=torch.Generator().manual_seed(seed), dtype=i32).cuda()
        adapters.append((s, synth.normal_bf16((T, K), 1.0, seed).cuda(), synth.normal_bf16((M, K), 0.05, seed + 1).cuda(),
                         synth.normal_bf16((n, r, K), 0.1, seed + 2).cuda(), synth.normal_bf16((n, M, r), 0.2, seed + 3).cuda(),
                         torch.ones(n, device="cuda"), ids, torch.empty(T, M, dtype=bf16, device="cuda"),
                         torch.zeros(1, dtype=i32, device="cuda"), B.new_adapter_workspace(s)))

    def step(q):
        shape, budget, off, inputs, b = q
        _router_step(inputs, b, shape, budget, off)

    for q in steps:
        step(q)
    for a in adapters:
        B.moe_adapter_linear(*a)
    torch.cuda.synchronize()
    want_steps, want_y = [{k: q[4][k].clone() for k in keys} for q in steps], [a[7].clone() for a in adapters]
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        for q in steps:
            for k in keys:
                q[4][k].fill_(3)
        for a in adapters:
            a[7].fill_(3)
        torch.cuda.synchronize()
        for _ in range(8):
            for q, s in zip(steps, streams):
                with torch.cuda.stream(s):
                    step(q)
            with torch.cuda.stream(streams[2]):
                for a in adapters:
                    B.moe_adapter_linear(*a)
        torch.cuda.synchronize()
        assert all(torch.equal(w[k], q[4][k]) for w, q in zip(want_steps, steps) for k in keys)
        assert all(torch.equal(w, a[7]) and int(a[8]) == 0 for w, a in zip(want_y, adapters))
