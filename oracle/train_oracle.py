"""The calls for training the layer, in fp64 numpy (formulas: include/allocmoe.h): ragged products, the routed experts' backward pass,
the norms around a block, AdamW with its 8-bit states.  Written from the definitions; nothing here is shared with the CUDA path."""
import numpy as np

BLOCK = 256


def segments(offsets):
    return [(int(a), int(b)) for a, b in zip(offsets, offsets[1:])]


def product(x, offsets, W, transposed=False):
    """y[p] = x[p] W_e^T (or x[p] W_e); rows outside every segment are zero."""
    out = np.zeros((x.shape[0], W.shape[2] if transposed else W.shape[1]))
    for e, (a, b) in enumerate(segments(offsets)):
        out[a:b] = x[a:b] @ (W[e] if transposed else W[e].T)
    return out


def weight_gradient(dy, x, offsets):
    return np.stack([dy[a:b].T @ x[a:b] for a, b in segments(offsets)])


def experts_forward(x, offsets, W13, W2):
    I = W2.shape[2]
    u = product(x, offsets, W13)
    return product(u[:, :I] / (1 + np.exp(-u[:, :I])) * u[:, I:], offsets, W2)


def experts_backward(x, offsets, W13, W2, dy):
    """(dx, dW13, dW2) for rows x of the list."""
    I = W2.shape[2]
    u = product(x, offsets, W13)
    u1, u3 = u[:, :I], u[:, I:]
    sg = 1 / (1 + np.exp(-u1))
    dh = product(dy, offsets, W2, transposed=True)
    du = np.concatenate([dh * u3 * sg * (1 + u1 * (1 - sg)), dh * u1 * sg], axis=1)
    return product(du, offsets, W13, transposed=True), weight_gradient(du, x, offsets), weight_gradient(dy, u1 * sg * u3, offsets)


def _sigmoid(g):
    return 1.0 if g is None else 1 / (1 + np.exp(-g))


def norm_r(r, y, w_post, gate, scale, eps, y_as_is=False):
    y_hat = y if y_as_is else y / np.sqrt((y * y).mean(1, keepdims=True) + eps)
    return r + scale * _sigmoid(gate) * (w_post * y_hat)


def norm_n(r, w_pre, eps):
    return w_pre * r / np.sqrt((r * r).mean(1, keepdims=True) + eps)


def norm_backward(r, y, w_post, gate, scale, w_pre, d_n, d_r_out, eps, y_as_is=False):
    """Gradients of norm_r followed by norm_n, with r the output of norm_r: a dict, and next to each value the sum of the magnitudes of
    its terms ("|name|"), which roundings are relative to."""
    out = {}
    rms_r = np.sqrt((r * r).mean(1, keepdims=True) + eps)
    r_hat, a = r / rms_r, d_n * w_pre
    out["d_r"] = d_r_out + (a - r_hat * (a * r_hat).mean(1, keepdims=True)) / rms_r
    out["|d_r|"] = np.abs(d_r_out) + (np.abs(a) + np.abs(r_hat) * np.abs(a * r_hat).mean(1, keepdims=True)) / rms_r
    out["dw_pre"], out["|dw_pre|"] = (d_n * r_hat).sum(0), np.abs(d_n * r_hat).sum(0)
    if y is None:
        return out
    rms_y = np.ones_like(rms_r) if y_as_is else np.sqrt((y * y).mean(1, keepdims=True) + eps)
    y_hat, sg = y / rms_y, _sigmoid(gate)
    d_p, m_p = out["d_r"] * scale * sg, out["|d_r|"] * np.abs(scale) * sg
    b, m_b = d_p * w_post, m_p * np.abs(w_post)
    back = 0.0 if y_as_is else y_hat * (b * y_hat).mean(1, keepdims=True)
    m_back = 0.0 if y_as_is else np.abs(y_hat) * (m_b * np.abs(y_hat)).mean(1, keepdims=True)
    out["d_y"], out["|d_y|"] = (b - back) / rms_y, (m_b + m_back) / rms_y
    out["dw_post"], out["|dw_post|"] = (d_p * y_hat).sum(0), (m_p * np.abs(y_hat)).sum(0)
    t, m_t = out["d_r"] * sg * w_post * y_hat, out["|d_r|"] * sg * np.abs(w_post * y_hat)
    out["d_scale"], out["|d_scale|"] = t.sum(), m_t.sum()
    if gate is not None:
        d, m = t * scale * (1 - sg), m_t * np.abs(scale) * (1 - sg)
        if gate.shape[1] == 1:
            d, m = d.sum(1, keepdims=True), m.sum(1, keepdims=True)
        out["d_gate"], out["|d_gate|"] = d, m
    return out


def adamw(p, g, m, v, lr, bias1, bias2, clip, beta1, beta2, eps, decay):
    g = g * clip
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * decay) - lr * (m / bias1) / (np.sqrt(v / bias2) + eps), m, v


def moments_fp32(g, m, v, clip, beta1, beta2):
    """m and v as the operator defines them: each fp32 operation rounded by itself."""
    f = np.float32
    g = g.astype(f) * f(clip)
    m = m.astype(f) * f(beta1) + g * f(1 - beta1)
    v = v.astype(f) * f(beta2) + (g * f(1 - beta2)) * g
    return m, v


def _blocks(a):
    n = a.size
    return np.pad(a.astype(np.float32), (0, -n % BLOCK)).reshape(-1, BLOCK)


def _scale(largest, top):
    used = largest >= np.float32(2.0 ** -100)
    safe = np.where(used, largest, np.float32(1))
    return np.where(used, safe / np.float32(top), np.float32(0)), np.where(used, np.float32(top) / safe, np.float32(0))


# the 127 values of e4m3 from zero up, by code: exponent 4 bits (bias 7), mantissa 3, no infinities
E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def m_codes(m):
    """(codes, scales): e4m3, nearest, ties to the even code."""
    b = _blocks(m)
    scale, factor = _scale(np.abs(b).max(1, keepdims=True), 448.0)
    x = (b * factor).astype(np.float64)
    lo = np.clip(np.searchsorted(E4M3, np.abs(x), side="right") - 1, 0, 125)
    below, above = np.abs(x) - E4M3[lo], E4M3[lo + 1] - np.abs(x)
    code = np.where((above < below) | ((above == below) & (lo % 2 == 1)), lo + 1, lo)
    code = (code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)
    return code.reshape(-1)[:m.size], scale.reshape(-1)


def m_values(codes, scale):
    mag = np.append(E4M3, 0.0)[codes & 127].astype(np.float32)
    return np.where(codes >= 128, -mag, mag) * np.repeat(scale, BLOCK)[:codes.size]


V_VALUES = np.array([0.0] + [(1 + c % 16 / 16) * 2.0 ** (c // 16 - 15) for c in range(1, 256)])


def v_codes(v):
    """(codes, scales) of sqrt(v): nearest of V_VALUES among normal numbers, ties to the even mantissa, at least 1 above zero."""
    b = np.sqrt(_blocks(v))
    scale, factor = _scale(b.max(1, keepdims=True), 1.9375)
    x = (b * factor).astype(np.float64)
    frac, exp = np.frexp(np.where(x > 0, x, 1.0))            # x = frac 2^exp, frac in [0.5, 1)
    code = np.rint((2 * frac - 1) * 16).astype(np.int64) + (exp - 1 + 15) * 16
    code = np.where((b > 0) & (scale > 0), np.clip(code, 1, 255), 0).astype(np.uint8)
    return code.reshape(-1)[:v.size], scale.reshape(-1)


def v_values(codes, scale):
    u = V_VALUES[codes].astype(np.float32) * np.repeat(scale, BLOCK)[:codes.size]
    return u * u
