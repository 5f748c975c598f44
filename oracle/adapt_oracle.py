"""Plain fp64 CPU forms of the calls that adapt a frozen layer: the balance loss and its counts, the gate's and the
combine step's gradients, projections with low-rank adapters.  Written from the formulas, row by row."""
from __future__ import annotations

import numpy as np


def sequences(seq_offsets, T):
    """The packed sequences as (first row, end) pairs."""
    if seq_offsets is None:
        return [(0, T)]
    return [(int(a), int(b)) for a, b in zip(seq_offsets[:-1], seq_offsets[1:])]


def balance_loss(scores, topk_idx, n_sel, seq_offsets, alpha):
    """(counts [B,N] int, coef [B,N], loss): loss = alpha/B sum_b sum_i (N c/C) mean_t s, coef its derivative by s."""
    s = np.asarray(scores, np.float64)
    T, N = s.shape
    K = topk_idx.shape[1]
    seqs = sequences(seq_offsets, T)
    counts = np.zeros((len(seqs), N), np.int64)
    coef = np.zeros((len(seqs), N))
    loss = 0.0
    for b, (lo, hi) in enumerate(seqs):
        for t in range(lo, hi):
            n = K if n_sel is None else min(max(int(n_sel[t]), 0), K)
            for j in range(n):
                counts[b, topk_idx[t, j]] += 1
        C = counts[b].sum()
        if C == 0:
            continue
        coef[b] = alpha / len(seqs) * N * counts[b] / C / (hi - lo)
        loss += (coef[b] * s[lo:hi].sum(0)).sum()
    return counts, coef, loss


def balance_loss_of_logits(logits, topk_idx, n_sel, seq_offsets, alpha):
    """The loss as a function of the logits, the selection held fixed (for difference quotients)."""
    z = np.asarray(logits, np.float64)
    e = np.exp(z - z.max(1, keepdims=True))
    return balance_loss(e / e.sum(1, keepdims=True), topk_idx, n_sel, seq_offsets, alpha)[2]


def score_gradient(T, N, topk_idx, n_sel, d_topk_score, coef, seq_offsets):
    """g [T,N] and the same sum of absolute values; rows outside every sequence hold zeros."""
    g, g_abs = np.zeros((T, N)), np.zeros((T, N))
    for b, (lo, hi) in enumerate(sequences(seq_offsets, T)):
        for t in range(lo, hi):
            if coef is not None:
                g[t] += np.asarray(coef[b], np.float64)
                g_abs[t] += np.abs(np.asarray(coef[b], np.float64))
            if d_topk_score is not None:
                K = topk_idx.shape[1]
                n = K if n_sel is None else min(max(int(n_sel[t]), 0), K)
                for j in range(n):
                    g[t, topk_idx[t, j]] += float(d_topk_score[t, j])
                    g_abs[t, topk_idx[t, j]] += abs(float(d_topk_score[t, j]))
    return g, g_abs


def gate_backward(x, W_gate, scores, topk_idx, n_sel, d_topk_score, coef, seq_offsets):
    """(d_logits, dx, dW, d_bias) in fp64; x / W_gate may be None (their products are then None)."""
    s = np.asarray(scores, np.float64)
    T, N = s.shape
    g, _ = score_gradient(T, N, topk_idx, n_sel, d_topk_score, coef, seq_offsets)
    d = np.zeros((T, N))
    for lo, hi in sequences(seq_offsets, T):
        d[lo:hi] = s[lo:hi] * (g[lo:hi] - (s[lo:hi] * g[lo:hi]).sum(1, keepdims=True))
    dx = None if W_gate is None else d @ np.asarray(W_gate, np.float64).T
    dW = None
    if x is not None:
        dW = np.zeros((x.shape[1], N))
        for lo, hi in sequences(seq_offsets, T):
            dW += np.asarray(x[lo:hi], np.float64).T @ d[lo:hi]
    return d, dx, dW, d.sum(0)


def combine_backward(d_out, y_perm, pair_pos, topk_score, n_sel, d_y_perm):
    """(d_topk_score, d_y_perm): d_y_perm is the buffer's earlier content, rows that no pair names keep it."""
    d_out, y = np.asarray(d_out, np.float64), np.asarray(y_perm, np.float64)
    T, K = pair_pos.shape
    d_score, d_y = np.zeros((T, K)), np.array(d_y_perm, np.float64)
    for t in range(T):
        for j in range(min(int(n_sel[t]), K)):
            p = int(pair_pos[t, j])
            if 0 <= p < y.shape[0]:
                d_score[t, j] = (d_out[t] * y[p]).sum()
                d_y[p] = float(topk_score[t, j]) * d_out[t]
    return d_score, d_y


def adapter_linear(x, W, A, B, scale, adapter_id):
    """y = x W^T + scale[a] (x A_a^T) B_a^T, a = adapter_id[t]; rows with a outside [0, n) get the projection alone."""
    x, A, B = (np.asarray(v, np.float64) for v in (x, A, B))
    y = x @ np.asarray(W, np.float64).T
    for a in range(A.shape[0]):
        t = np.nonzero(np.asarray(adapter_id) == a)[0]
        if len(t):
            y[t] += float(scale[a]) * ((x[t] @ A[a].T) @ B[a].T)
    return y


def shared_ffn_adapted(x, Wsh13, Wsh2, A13, B13, A2, B2, scale, adapter_id):
    """The S shared experts as one block with adapters beside both projections (fp64 throughout)."""
    S, two_i, H = Wsh13.shape
    I = two_i // 2
    u = adapter_linear(x, np.asarray(Wsh13).reshape(S * two_i, H), A13, B13, scale, adapter_id).reshape(-1, S, 2, I)
    gate, up = u[:, :, 0], u[:, :, 1]
    h = (gate / (1.0 + np.exp(-gate)) * up).reshape(-1, S * I)
    W2 = np.concatenate(list(np.asarray(Wsh2)), axis=1)
    return adapter_linear(h, W2, A2, B2, scale, adapter_id), h
