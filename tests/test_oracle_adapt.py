"""The fp64 forms of the router's gradients and the adapters, against difference quotients and independent forms."""
import numpy as np
import pytest

from oracle import adapt_oracle as ado
from oracle import alloc_moe_oracle as orc


def _case(T, N, K, seed, offsets=None):
    r = np.random.default_rng(seed)
    logits = r.normal(size=(T, N))
    s = orc.softmax_scores(logits).astype(np.float64)
    idx = np.argsort(-s, axis=1, kind="stable")[:, :K].astype(np.int32)
    n_sel = r.integers(0, K + 1, size=T).astype(np.int32)
    return r, logits, s, idx, n_sel, offsets


CASES = [(5, 8, 3, None), (9, 12, 2, [0, 4, 9]), (9, 8, 3, [1, 1, 6, 8]), (1, 8, 1, None), (6, 8, 8, [0, 6])]


@pytest.mark.parametrize("T,N,K,off", CASES)
def test_balance_gradient_is_the_losss_difference_quotient(T, N, K, off):
    r, logits, s, idx, n_sel, off = _case(T, N, K, 11 + T, off)
    e = np.exp(logits - logits.max(1, keepdims=True))
    s = e / e.sum(1, keepdims=True)
    counts, coef, loss = ado.balance_loss(s, idx, n_sel, off, 0.7)
    d = ado.gate_backward(None, None, s, None, None, None, coef, off)[0]
    h = 1e-5
    for t in range(T):
        for i in range(N):
            z = logits.copy()
            z[t, i] += h
            up = ado.balance_loss_of_logits(z, idx, n_sel, off, 0.7)
            z[t, i] -= 2 * h
            dn = ado.balance_loss_of_logits(z, idx, n_sel, off, 0.7)
            # central difference: truncation h^2 |f'''| / 6 (f''' <= loss) and cancellation 2^-53 loss / h
            assert abs((up - dn) / (2 * h) - d[t, i]) <= 2e-10 * max(loss, 1.0) + 1e-9 * abs(d[t, i]), (t, i)


def test_balance_loss_is_alpha_when_balanced_and_skips_empty_sequences():
    N, T = 8, 16
    s = np.full((T, N), 1.0 / N)
    idx = np.stack([(np.arange(T) + j) % N for j in range(2)], axis=1)
    c, coef, loss = ado.balance_loss(s, idx, None, None, 0.25)
    assert (c == 4).all() and abs(loss - 0.25) < 1e-12
    c, coef, loss = ado.balance_loss(s, idx, np.zeros(T, int), None, 0.25)
    assert c.sum() == 0 and loss == 0 and (coef == 0).all()
    c, coef, loss = ado.balance_loss(s, idx, None, [0, 8, 8, 16], 0.25)     # the empty one counts in 1 / n_seq only
    assert abs(loss - 0.25 * 2 / 3) < 1e-12 and (coef[1] == 0).all()


@pytest.mark.parametrize("T,N,K,off", CASES)
def test_gate_backward_is_the_difference_quotient_of_a_weighted_score_sum(T, N, K, off):
    r, _, _, idx, n_sel, off = _case(T, N, K, 5 + T, off)
    H = 6
    x, W, bias = r.normal(size=(T, H)), r.normal(size=(H, N)), r.normal(size=N)
    d_top = r.normal(size=(T, K))
    inside = np.zeros(T, bool)
    for lo, hi in ado.sequences(off, T):
        inside[lo:hi] = True

    def f(x, W, bias):
        z = x @ W + bias
        e = np.exp(z - z.max(1, keepdims=True))
        s = e / e.sum(1, keepdims=True)
        v = 0.0
        for t in range(T):
            for j in range(n_sel[t] if inside[t] else 0):
                v += d_top[t, j] * s[t, idx[t, j]]
        return v, s

    _, s = f(x, W, bias)
    d, dx, dW, db = ado.gate_backward(x, W, s, idx, n_sel, d_top, None, off)
    h = 1e-5
    for arr, grad in ((x, dx), (W, dW), (bias, db)):
        for q in range(arr.size):
            k = np.unravel_index(q, arr.shape)
            keep = arr[k]
            arr[k] = keep + h
            up = f(x, W, bias)[0]
            arr[k] = keep - h
            dn = f(x, W, bias)[0]
            arr[k] = keep
            assert abs((up - dn) / (2 * h) - grad[k]) <= 1e-7 * (1 + abs(grad[k]))


def test_combine_backward_matches_difference_quotients():
    r = np.random.default_rng(3)
    T, K, H, Bn = 4, 3, 8, 7
    y, w, n_sel = r.normal(size=(Bn, H)), r.random((T, K)), np.array([3, 0, 2, 1])
    pos = np.full((T, K), -1)
    pos[np.arange(K)[None, :] < n_sel[:, None]] = r.permutation(Bn)[:6]
    d_out = r.normal(size=(T, H))

    def f(w, y):
        return sum(w[t, j] * (d_out[t] * y[pos[t, j]]).sum() for t in range(T) for j in range(n_sel[t]))

    d_score, d_y = ado.combine_backward(d_out, y, pos, w, n_sel, np.zeros_like(y))
    for arr, grad in ((w, d_score), (y, d_y)):
        for q in range(arr.size):
            k = np.unravel_index(q, arr.shape)
            keep = arr[k]
            arr[k] = keep + 0.5
            up = f(w, y)
            arr[k] = keep - 0.5
            dn = f(w, y)
            arr[k] = keep
            assert abs(up - dn - grad[k]) <= 1e-12 * (1 + abs(grad[k]))      # linear in both


def test_adapter_linear_is_the_projection_by_the_merged_weight():
    r = np.random.default_rng(8)
    x, W = r.normal(size=(7, 10)), r.normal(size=(6, 10))
    A, B, scale = r.normal(size=(3, 2, 10)), r.normal(size=(3, 6, 2)), np.array([0.5, 2.0, 1.0])
    ids = np.array([0, -1, 2, 2, 1, 5, 0])
    y = ado.adapter_linear(x, W, A, B, scale, ids)
    for t, a in enumerate(ids):
        merged = W + (scale[a] * B[a] @ A[a] if 0 <= a < 3 else 0)
        assert np.allclose(y[t], merged @ x[t], rtol=1e-12, atol=1e-12)


def test_shared_ffn_adapted_without_adapters_is_the_shared_experts():
    r = np.random.default_rng(9)
    T, H, I, S = 5, 8, 4, 2
    x, W13, W2 = r.normal(size=(T, H)), r.normal(size=(S, 2 * I, H)), r.normal(size=(S, H, I))
    A13, B13 = r.normal(size=(1, 2, H)), r.normal(size=(1, S * 2 * I, 2))
    A2, B2 = r.normal(size=(1, 2, S * I)), r.normal(size=(1, H, 2))
    y, _ = ado.shared_ffn_adapted(x, W13, W2, A13, B13, A2, B2, np.ones(1), np.full(T, -1))
    want = np.zeros((T, H))
    for s in range(S):
        a, b = x @ W13[s, :I].T, x @ W13[s, I:].T
        want += (a / (1 + np.exp(-a)) * b) @ W2[s].T
    assert np.allclose(y, want, rtol=1e-12, atol=1e-12)
