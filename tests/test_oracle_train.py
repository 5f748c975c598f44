"""The fp64 forms of the training calls against differences of their forward forms, and the 8-bit formats against their definitions."""
import numpy as np
import pytest

from oracle import train_oracle as orc

EPS = 1e-6


def _slope(f, at, step=1e-6):
    """d f / d at, by central differences."""
    out = np.zeros_like(at)
    for i in np.ndindex(at.shape):
        keep = at[i]
        at[i] = keep + step
        hi = f()
        at[i] = keep - step
        lo = f()
        at[i] = keep
        out[i] = (hi - lo) / (2 * step)
    return out


def test_products_and_their_gradients():
    rng = np.random.default_rng(0)
    off = [1, 1, 4, 6]
    x, W, dy = rng.normal(size=(7, 3)), rng.normal(size=(3, 4, 3)), rng.normal(size=(7, 4))
    f = lambda: (dy * orc.product(x, off, W)).sum()
    assert np.allclose(orc.product(dy, off, W, transposed=True), _slope(f, x), atol=1e-7)
    assert np.allclose(orc.weight_gradient(dy, x, off), _slope(f, W), atol=1e-7)
    assert not orc.product(x, off, W)[[0, 6]].any() and not orc.weight_gradient(dy, x, off)[0].any()


def test_experts_backward():
    rng = np.random.default_rng(1)
    off = [0, 2, 2, 5]
    x, W13, W2, dy = rng.normal(size=(5, 4)), rng.normal(size=(3, 6, 4)), rng.normal(size=(3, 4, 3)), rng.normal(size=(5, 4))
    f = lambda: (dy * orc.experts_forward(x, off, W13, W2)).sum()
    got = orc.experts_backward(x, off, W13, W2, dy)
    for g, at in zip(got, (x, W13, W2)):
        assert np.allclose(g, _slope(f, at), atol=1e-6)


@pytest.mark.parametrize("gate_cols", [0, 1, 5])
@pytest.mark.parametrize("y_as_is", [False, True])
def test_norm_backward(gate_cols, y_as_is):
    rng = np.random.default_rng(2)
    T, H = 3, 5
    r, y, wp, wn = rng.normal(size=(T, H)), rng.normal(size=(T, H)), rng.normal(size=H), rng.normal(size=H)
    gate = rng.normal(size=(T, gate_cols)) if gate_cols else None
    dn, dr, scale = rng.normal(size=(T, H)), rng.normal(size=(T, H)), np.array([0.7])

    def f():
        out = orc.norm_r(r, y, wp, gate, scale[0], EPS, y_as_is)
        return (dr * out).sum() + (dn * orc.norm_n(out, wn, EPS)).sum()

    got = orc.norm_backward(orc.norm_r(r, y, wp, gate, scale[0], EPS, y_as_is), y, wp, gate, scale[0], wn, dn, dr, EPS, y_as_is)
    for name, at in (("d_r", r), ("d_y", y), ("dw_post", wp), ("dw_pre", wn), ("d_scale", scale), ("d_gate", gate)):
        if at is not None:
            assert np.allclose(got[name], _slope(f, at), atol=1e-6), name
            assert (np.abs(got[name]) <= got["|" + name + "|"] * (1 + 1e-12) + 1e-12).all(), name


def test_adamw_first_steps_by_hand():
    p, m, v = orc.adamw(np.array([1.0]), np.array([2.0]), np.array([0.0]), np.array([0.0]), 0.1, 0.1, 0.01, 1.0, 0.9, 0.99, 0.0, 0.5)
    assert np.allclose([p[0], m[0], v[0]], [1 * 0.95 - 0.1, 0.2, 0.04])


def test_m_codes_are_the_nearest_values():
    rng = np.random.default_rng(3)
    m = (rng.normal(size=1000) * np.exp(rng.normal(size=1000) * 3)).astype(np.float32)
    m[256:512] = 0
    codes, scale = orc.m_codes(m)
    got, b = orc.m_values(codes, scale), np.repeat(scale, 256)[:1000]
    assert not got[256:512].any() and scale[1] == 0
    # the nearest value, but for the four fp32 roundings on the way there and back (scale, factor, and the two products)
    for i in list(range(256)) + list(range(512, 1000)):
        nearest = np.abs(np.concatenate([-orc.E4M3, orc.E4M3]) * b[i] - m[i]).min()
        assert abs(got[i] - m[i]) <= nearest + 4 * 2.0 ** -24 * max(abs(m[i]), abs(got[i]))


def test_v_codes_keep_what_is_above_zero():
    rng = np.random.default_rng(4)
    v = (rng.normal(size=777).astype(np.float32) ** 2) * np.exp(rng.normal(size=777) * 4).astype(np.float32)
    v[::5] = 0
    v[1] = 1e-25
    codes, scale = orc.v_codes(v)
    assert ((codes > 0) == (v > 0)).all() and codes.max() == 255
    u, x = np.sqrt(orc.v_values(codes, scale)), np.sqrt(v.astype(np.float64))
    big = codes > 16
    assert (np.abs(u - x)[big] <= x[big] * (2.0 ** -5 + 4 * 2.0 ** -24)).all()      # half a step of four mantissa bits, and the fp32 roundings
    assert (np.diff(orc.V_VALUES) > 0).all()


def test_v_ties_go_to_the_even_code():
    v = np.zeros(256, np.float32)
    v[0] = 1.9375 ** 2
    v[1], v[2] = (1 + 1 / 32) ** 2, (1 + 3 / 32) ** 2
    codes, _ = orc.v_codes(v)
    assert codes[0] == 255 and codes[1] == 240 and codes[2] == 242
