"""Projections with low-rank adapters per request, and the shared experts with them, against the fp64 oracle.

Tolerances come from counting roundings (u = 2^-24 for fp32 sums of n terms: n u of the absolute terms; 2^-8 for a
rounding to bf16) and are built element by element in _bound and test_shared_ffn_adapted."""
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


def _np(t):
    return t.detach().double().cpu().numpy()


def _ids(kind, T, n, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "none":
        return torch.full((T,), -1, dtype=i32)
    if kind == "one":
        return torch.full((T,), n - 1, dtype=i32)
    if kind == "own":                                          # every token another adapter, as far as they go
        return (torch.randperm(T, generator=g) % n).to(i32)
    if kind == "mixed":                                        # any order, some tokens without one
        return torch.randint(-1, n, (T,), generator=g, dtype=i32)
    if kind == "sparse":                                       # few tokens of a batch have an adapter
        ids = torch.full((T,), -3, dtype=i32)
        ids[torch.randperm(T, generator=g)[:max(1, T // 17)]] = 0
        return ids
    assert kind == "runs"                                      # requests one behind the other, every fourth without one
    cuts = sorted(torch.randint(0, T + 1, (6,), generator=g).tolist())
    ids = torch.zeros(T, dtype=i32)
    for k, (a, b) in enumerate(zip([0] + cuts, cuts + [T])):
        ids[a:b] = -1 if k % 4 == 3 else k % n
    return ids


def _inputs(T, K, M, n, r, seed):
    return dict(x=synth.normal_bf16((T, K), 1.0, seed), W=synth.normal_bf16((M, K), 0.05, seed + 1),
                A=synth.normal_bf16((n, r, K), K ** -0.5, seed + 2), Bm=synth.normal_bf16((n, M, r), 0.2, seed + 3),
                scale=torch.tensor([(0.5, 1.0, -2.0, 1.75)[i % 4] for i in range(n)]))


def _call(T, K, M, n, r, d, ids, fill=-7.0):
    s = B.make_adapter_shape(T, K, M, n, r)
    y = torch.full((T, M), fill, dtype=bf16, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    ws = B.new_adapter_workspace(s)
    ws.fill_(255)
    B.moe_adapter_linear(s, d["x"].cuda(), d["W"].cuda(), d["A"].cuda(), d["Bm"].cuda(), d["scale"].cuda(), ids.cuda(), y, st, ws)
    torch.cuda.synchronize()
    return y, int(st.item())


def _bound(x, W, A, Bm, scale, ids, y, e_x=None):
    """Error bound of the adapted projection for inputs x known to within e_x (before y's own rounding is added)."""
    x, W, A, Bm = np.abs(x), np.abs(W), np.abs(A), np.abs(Bm)
    K = x.shape[1]
    e_x = np.zeros_like(x) if e_x is None else e_x
    e = e_x @ W.T + (K + 8) * U * (x @ W.T)
    for a in range(A.shape[0]):
        t = np.nonzero(ids == a)[0]
        if len(t):
            s = abs(float(scale[a]))
            v = s * (x[t] @ A[a].T)                                    # an upper bound of |v|
            e_v = s * (e_x[t] @ A[a].T) + (K + 8) * U * v
            v_val = v                                                  # bf16 rounding of v: 2^-8 of |v| <= this bound
            e[t] += e_v @ Bm[a].T + (UB + (A.shape[1] + 8) * U) * ((v_val + e_v) @ Bm[a].T)
    return e


def _check(d, ids, y, rows=None):
    ids = ids.numpy()
    rows = np.arange(len(ids)) if rows is None else rows
    x, W, A, Bm, sc = _np(d["x"])[rows], _np(d["W"]), _np(d["A"]), _np(d["Bm"]), _np(d["scale"])
    want = ado.adapter_linear(x, W, A, Bm, sc, ids[rows])
    # v's rounding is bounded by its actual value where that is known
    e = (x.shape[1] + 8) * U * (np.abs(x) @ np.abs(W).T)
    for a in range(A.shape[0]):
        t = np.nonzero(ids[rows] == a)[0]
        if len(t):
            v = sc[a] * (x[t] @ A[a].T)
            e_v = (x.shape[1] + 8) * U * abs(sc[a]) * (np.abs(x[t]) @ np.abs(A[a]).T)
            e[t] += (UB * np.abs(v) + (1 + UB) * e_v) @ np.abs(Bm[a]).T
            e[t] += (A.shape[1] + 8) * U * (np.abs(v) @ np.abs(Bm[a]).T)
    got = _np(y)[rows]
    assert np.all(np.abs(got - want) <= (1 + UB) * e + UB * np.abs(want)), \
        "worst %.3g of its bound" % (np.abs(got - want) / ((1 + UB) * e + UB * np.abs(want))).max()


# T, K, M, n_adapters, rank: one token, tiles that end inside, sizes that are no multiple of a tile in any direction, the
# smallest and the largest rank, more adapters than tokens
CASES = [
    (1, 64, 64, 1, 8), (1, 2048, 4096, 4, 16), (2, 8, 8, 3, 8), (7, 136, 72, 5, 24), (31, 512, 264, 40, 16), (63, 72, 1000, 9, 64),
    (64, 2048, 2816, 48, 16), (65, 1408, 320, 3, 128), (127, 256, 200, 200, 32), (128, 520, 512, 2, 40), (129, 256, 256, 7, 16),
    (200, 1000, 136, 64, 72), (300, 640, 1096, 17, 120), (513, 128, 2048, 3, 64), (1100, 384, 408, 30, 8), (1030, 2048, 256, 5, 128),
    # enough tiles for every tile width: 160, 192, 224 and 256 weight rows
    (2443, 128, 2272, 7, 56), (4000, 64, 2816, 5, 32), (2045, 64, 2048, 3, 16), (3000, 72, 4096, 4, 8),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T%d-K%d-M%d-n%d-r%d" % c)
@pytest.mark.parametrize("kind", ["none", "one", "own", "mixed", "sparse", "runs"])
def test_adapter_linear(case, kind):
    T, K, M, n, r = case
    d, ids = _inputs(T, K, M, n, r, 5), _ids(kind, T, n, T)
    y, st = _call(T, K, M, n, r, d, ids)
    assert st == 0
    _check(d, ids, y)


@pytest.mark.parametrize("T,K,M,n,r,kind", [(64, 4096, 14336, 3, 16, "mixed"), (2500, 2048, 1408, 6, 64, "runs"),
                                            (4096, 1024, 2816, 64, 16, "mixed"), (1, 14336, 4096, 2, 64, "one")])
def test_adapter_linear_at_size(T, K, M, n, r, kind):
    """Full-size products; a seeded choice of rows is compared (every 128-row block has some)."""
    d, ids = _inputs(T, K, M, n, r, 6), _ids(kind, T, n, 3)
    y, st = _call(T, K, M, n, r, d, ids)
    assert st == 0
    rows = np.unique(np.concatenate([np.arange(0, T, 61), [T - 1], np.arange(max(0, T - 130), T, 43)]))
    _check(d, ids, y, rows)
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("T,K,M,n,r", [(40, 256, 264, 6, 16), (128, 128, 128, 6, 64), (700, 256, 520, 6, 16), (1500, 128, 256, 6, 128)])
@pytest.mark.parametrize("what", ["A", "B", "Binf", "x", "scale", "unused"])
def test_one_requests_broken_values_stay_its_own(T, K, M, n, r, what):
    """NaN or infinities in one adapter, or in one token, reach no row of another request."""
    d, ids = _inputs(T, K, M, n, r, 8), _ids("mixed", T, n - 1, 4)      # adapter n - 1 is named by no token
    clean, _ = _call(T, K, M, n, r, d, ids)
    bad = {k: v.clone() for k, v in d.items()}
    touched = ids == 2
    if what == "A":
        bad["A"][2, 3] = float("nan")
    elif what == "B":
        bad["Bm"][2, M // 2:, r - 1] = float("nan")
    elif what == "Binf":
        bad["Bm"][2, :5, 0] = float("inf")
    elif what == "x":
        touched = torch.zeros(T, dtype=torch.bool)
        touched[T // 3] = touched[T - 1] = True
        bad["x"][touched] = float("nan")
    elif what == "scale":
        bad["scale"][2] = float("inf")
    else:
        bad["A"][n - 1], bad["Bm"][n - 1], bad["scale"][n - 1] = float("nan"), float("inf"), float("nan")
        touched[:] = False
    y, st = _call(T, K, M, n, r, bad, ids)
    assert st == 0
    assert torch.equal(y.cpu()[~touched].view(torch.int16), clean.cpu()[~touched].view(torch.int16))
    if what == "B":                                             # its own rows are what the formula gives, column by column
        assert torch.isnan(y.cpu()[touched][:, M // 2:]).all()
        _check({**d, "W": d["W"][:M // 2], "Bm": d["Bm"][:, :M // 2]}, ids, y[:, :M // 2].contiguous())
    if what in ("A", "x"):
        assert torch.isnan(y.cpu()[touched]).all()


def test_ids_beyond_the_adapters_are_reported_and_get_the_projection_alone():
    for T in (50, 700):
        K, M, n, r = 128, 192, 4, 16
        d, ids = _inputs(T, K, M, n, r, 9), _ids("mixed", T, n, 5)
        bad = ids.clone()
        bad[::9] = n
        bad[1::9] = 2 ** 31 - 1
        bad[2::9] = -2 ** 31
        y, st = _call(T, K, M, n, r, d, bad)
        assert st == 1 << B.MOE_ERR_ARG
        as_none = torch.where((bad < 0) | (bad >= n), -1, bad)
        y2, st2 = _call(T, K, M, n, r, d, as_none)
        assert st2 == 0 and torch.equal(y.view(torch.int16), y2.view(torch.int16))


def test_rows_do_not_depend_on_their_neighbours_or_the_run():
    """The same token gives the same bits wherever it stands among the tokens of a batch, and on every run."""
    T, K, M, n, r = 100, 512, 264, 10, 16
    d, ids = _inputs(T, K, M, n, r, 10), _ids("mixed", T, n, 6)
    y, _ = _call(T, K, M, n, r, d, ids)
    perm = torch.randperm(T, generator=torch.Generator().manual_seed(1))
    y2, _ = _call(T, K, M, n, r, {**d, "x": d["x"][perm].contiguous()}, ids[perm].contiguous())
    assert torch.equal(y.cpu()[perm].view(torch.int16), y2.cpu().view(torch.int16))
    for _ in range(3):
        y3, _ = _call(T, K, M, n, r, d, ids, fill=9.0)
        assert torch.equal(y.view(torch.int16), y3.view(torch.int16))


# ------------------------------------------------------------------------------------------------ shared experts
def _shared_inputs(T, H, I, S, n, r, seed):
    return dict(x=synth.normal_bf16((T, H), 1.0, seed), W13=synth.normal_bf16((S, 2 * I, H), 0.05, seed + 1),
                W2=synth.normal_bf16((S, H, I), 0.05, seed + 2), A13=synth.normal_bf16((n, r, H), H ** -0.5, seed + 3),
                B13=synth.normal_bf16((n, S * 2 * I, r), 0.2, seed + 4),
                A2=synth.normal_bf16((n, r, S * I), (S * I) ** -0.5, seed + 5), B2=synth.normal_bf16((n, H, r), 0.2, seed + 6),
                scale=torch.tensor([(0.5, 1.0, -2.0)[i % 3] for i in range(n)]))


def _shared_call(T, H, I, S, d, ids, y=None, ws=None, st=None):
    shape = B.make_shape(T, H, 8, I, S, 1, 0)
    n, r = d["A13"].shape[:2]
    y = torch.full((T, H), -7.0, dtype=bf16, device="cuda") if y is None else y
    st = torch.zeros(1, dtype=i32, device="cuda") if st is None else st
    if ws is None:
        ws = B.new_shared_adapted_workspace(shape, n, r)
        ws.fill_(255)
    c = {k: v.cuda() for k, v in d.items()}
    B.moe_shared_ffn_adapted(shape, c["x"], c["W13"], c["W2"], c["A13"], c["B13"], c["A2"], c["B2"], c["scale"], ids.cuda(), y, st,
                             ws)
    torch.cuda.synchronize()
    return y, int(st.item())


SHARED = [(1, 64, 64, 1, 1, 8), (1, 2048, 1408, 2, 4, 16), (5, 128, 192, 3, 9, 16), (64, 256, 320, 2, 32, 32), (129, 192, 64, 1, 4, 64),
          (300, 320, 448, 2, 5, 128), (700, 512, 192, 2, 3, 16), (1025, 128, 128, 1, 40, 24),
          (2443, 64, 1408, 2, 4, 16)]


@pytest.mark.parametrize("case", SHARED, ids=lambda c: "T%d-H%d-I%d-S%d-n%d-r%d" % c)
@pytest.mark.parametrize("kind", ["none", "one", "mixed", "runs"])
def test_shared_ffn_adapted(case, kind):
    T, H, I, S, n, r = case
    d, ids = _shared_inputs(T, H, I, S, n, r, 12), _ids(kind, T, n, 7)
    y, st = _shared_call(T, H, I, S, d, ids)
    assert st == 0
    f = {k: _np(v) for k, v in d.items()}
    want, h = ado.shared_ffn_adapted(f["x"], f["W13"], f["W2"], f["A13"], f["B13"], f["A2"], f["B2"], f["scale"], ids.numpy())
    # u: the adapted projection's bound.  h = silu(u1) u3: |silu'| <= 1.1, |silu(u)| <= |u|; the fast exponential and divide
    # are good to 2^-20 for the |u| < 88 here; h rounds to bf16 once.  y: the second projection of an h known to within e_h.
    u = ado.adapter_linear(f["x"], f["W13"].reshape(-1, H), f["A13"], f["B13"], f["scale"], ids.numpy()).reshape(T, S, 2, I)
    e_u = _bound(f["x"], f["W13"].reshape(-1, H), f["A13"], f["B13"], f["scale"], ids.numpy(), None).reshape(T, S, 2, I)
    e1, e3 = e_u[:, :, 0], e_u[:, :, 1]
    e_h = (1.1 * e1 * (np.abs(u[:, :, 1]) + e3) + np.abs(u[:, :, 0]) * e3).reshape(T, S * I)
    e_h += (UB + 2.0 ** -20) * (np.abs(h) + e_h)
    W2 = np.concatenate(list(f["W2"]), axis=1)
    e = _bound(np.abs(h) + e_h, W2, f["A2"], f["B2"], f["scale"], ids.numpy(), None, e_h)
    assert np.all(np.abs(_np(y) - want) <= e + UB * (np.abs(want) + e))
    # and far tighter on average: independent roundings add up by their squares (2^-9.2 of a value each: h, v twice, y)
    rms = np.sqrt(((_np(y) - want) ** 2).mean() / max((want ** 2).mean(), 1e-30))
    assert rms <= 5e-3


def test_shared_ffn_adapted_without_adapters_equals_the_shared_experts_path():
    T, H, I, S = 96, 512, 256, 2
    d = _shared_inputs(T, H, I, S, 2, 16, 14)
    y, _ = _shared_call(T, H, I, S, d, torch.full((T,), -1, dtype=i32))
    shape = B.make_shape(T, H, 8, I, S, 1, 0)
    ref = torch.empty(T, H, dtype=bf16, device="cuda")
    st = torch.zeros(1, dtype=i32, device="cuda")
    B.moe_shared_ffn(shape, d["x"].cuda(), d["W13"].cuda(), d["W2"].cuda(), ref, st, B.new_workspace(shape, 0))
    torch.cuda.synchronize()
    a, b = _np(y), _np(ref)
    # both round h and y to bf16 once; their fp32 sums differ in order, which can flip roundings of h and of y
    assert np.abs(a - b).max() <= 4 * UB * np.abs(b).max() and np.sqrt(((a - b) ** 2).mean() / (b ** 2).mean()) <= 2e-3


def test_adapted_layer_from_tokens_to_output():
    """The layer with adapters on its shared experts: gate, routing, experts, adapted shared experts, combine."""
    cfg = synth.CONFIGS["c2"]
    T, H, N, I, S, K = 48, 256, 16, 128, 2, 4
    budget, shape = 100, B.make_shape(48, 256, 16, 128, 2, 4, 1)
    assert cfg.S == 2
    d, ids = _shared_inputs(T, H, I, S, 6, 16, 17), _ids("mixed", T, 6, 2)
    Wg = synth.normal_bf16((H, N), 0.05, 31).cuda()
    W13, W2 = synth.normal_bf16((N, 2 * I, H), 0.05, 32).cuda(), synth.normal_bf16((N, H, I), 0.05, 33).cuda()
    x = d["x"].cuda()
    z = lambda *s, dt=i32: torch.zeros(*s, dtype=dt, device="cuda")
    idx, top, n_sel, off, tok, wgt, pos = (z(T, K), z(T, K, dt=f32), z(T), z(N + 1), z(budget), z(budget, dt=f32), z(T, K))
    y_perm, out, st, ws = z(budget, H, dt=bf16), z(T, H, dt=bf16), z(1), B.new_workspace(shape, budget)
    B.moe_gate(shape, x, Wg, None, None, idx, top)
    B.moe_route(shape, idx, top, budget, n_sel, off, tok, wgt, pos, st)
    B.moe_grouped_ffn(shape, x, tok, off, budget, W13, W2, y_perm, st, ws)
    y_sh, _ = _shared_call(T, H, I, S, d, ids, st=st)
    B.moe_combine(shape, y_perm, pos, top, n_sel, y_sh, out)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    from oracle import alloc_moe_oracle as orc
    routed = orc.combine(_np(x).astype(np.float32), idx.cpu().numpy(), top.cpu().numpy(), n_sel.cpu().numpy(),
                         W13.float().cpu().numpy(), W2.float().cpu().numpy())
    f = {k: _np(v) for k, v in d.items()}
    shared, _ = ado.shared_ffn_adapted(f["x"], f["W13"], f["W2"], f["A13"], f["B13"], f["A2"], f["B2"], f["scale"], ids.numpy())
    want = routed + shared
    assert np.abs(_np(out) - want).max() <= 2e-2 * np.abs(want).max()


def test_adapter_calls_on_two_streams_and_from_a_graph():
    T, K, M, n, r = 64, 512, 1024, 16, 16
    s = B.make_adapter_shape(T, K, M, n, r)
    runs = []
    for seed in (1, 2):
        d, ids = _inputs(T, K, M, n, r, 50 + seed), _ids("mixed", T, n, seed).cuda()
        c = {k: v.cuda() for k, v in d.items()}
        runs.append((c, ids, torch.zeros(T, M, dtype=bf16, device="cuda"), torch.zeros(1, dtype=i32, device="cuda"),
                     B.new_adapter_workspace(s), torch.cuda.Stream()))

    def go(q, stream=None):
        c, ids, y, st, ws, _ = q
        B.moe_adapter_linear(s, c["x"], c["W"], c["A"], c["Bm"], c["scale"], ids, y, st, ws, stream=stream)

    ref = []
    for q in runs:
        go(q)
        torch.cuda.synchronize()
        ref.append(q[2].clone())
        q[2].zero_()
    torch.cuda.synchronize()
    for _ in range(20):                                         # each call has its workspace: they may overlap
        for q in runs:
            go(q, q[5])
    torch.cuda.synchronize()
    assert all(torch.equal(q[2], y) for q, y in zip(runs, ref))
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        go(runs[0])
        go(runs[1])
    for q in runs:
        q[2].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(q[2], y) for q, y in zip(runs, ref))
    runs[0][1].fill_(-1)                                        # other ids in the same buffer
    graph.replay()
    torch.cuda.synchronize()
    again = runs[0][2].clone()
    go(runs[0])
    torch.cuda.synchronize()
    assert torch.equal(again, runs[0][2]) and not torch.equal(again, ref[0])


def test_blocks_that_all_mix_adapters_give_the_same_bits_every_time():
    """Masked V of both CTAs of a pair in every tile, several tiles a pair: right, and the same on every run."""
    T, K, M, n, r = 4096, 128, 2816, 8, 64
    d, ids = _inputs(T, K, M, n, r, 61), (torch.arange(T) % n).to(i32)
    s = B.make_adapter_shape(T, K, M, n, r)
    c = {k: v.cuda() for k, v in d.items()}
    y, st, ws = (torch.empty(T, M, dtype=bf16, device="cuda"), torch.zeros(1, dtype=i32, device="cuda"), B.new_adapter_workspace(s))
    ids_gpu, first = ids.cuda(), None
    for _ in range(40):
        y.fill_(-7.0)
        B.moe_adapter_linear(s, c["x"], c["W"], c["A"], c["Bm"], c["scale"], ids_gpu, y, st, ws)
        first = y.clone() if first is None else first
        assert torch.equal(first.view(torch.int16), y.view(torch.int16))
    assert int(st.item()) == 0
    _check(d, ids, first, np.arange(0, T, 37))


def test_one_mixed_block_at_the_end_of_a_long_launch():
    """The warps that mask V wait for the one block that needs it through about 1.5e9 clocks of others: a launch's length
    alone is no timeout."""
    T, K, M, n, r = 1075 * 256, 131072, 74 * 256, 2, 8
    if torch.cuda.mem_get_info()[0] < 110 * 10 ** 9:
        pytest.skip("needs 90 GB")
    g = torch.Generator(device="cuda").manual_seed(3)
    z = lambda *s, std: torch.randn(*s, device="cuda", generator=g, dtype=bf16) * std
    rows = torch.tensor([0, 255, 256, T // 2, T - 256, T - 3, T - 2, T - 1], device="cuda")
    x = torch.zeros(T, K, dtype=bf16, device="cuda")
    x[rows] = z(len(rows), K, std=1.0)
    W, A, Bm = z(M, K, std=0.05), z(n, r, K, std=K ** -0.5), z(n, M, r, std=0.2)
    ids = torch.full((T,), -1, dtype=i32, device="cuda")
    ids[T - 2], ids[T - 1] = 1, 0
    scale, st = torch.tensor([1.0, -2.0], device="cuda"), torch.zeros(1, dtype=i32, device="cuda")
    s = B.make_adapter_shape(T, K, M, n, r)
    y, ws = torch.empty(T, M, dtype=bf16, device="cuda"), B.new_adapter_workspace(s)
    try:
        B.moe_adapter_linear(s, x, W, A, Bm, scale, ids, y, st, ws)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        got, xs = y[rows].double(), x[rows].double()
        untouched = torch.ones(T, dtype=torch.bool, device="cuda")
        untouched[rows] = False
        assert not y[untouched].any()
        for m in range(0, M, 1184):
            Wd = W[m:m + 1184].double()
            want, e = xs @ Wd.T, (K + 8) * U * (xs.abs() @ Wd.abs().T)
            for t, a in ((6, 1), (7, 0)):                    # as in _check, for the two tokens that have an adapter
                Bd = Bm[a, m:m + 1184].double()
                v, e_v = float(scale[a]) * (xs[t] @ A[a].double().T), (K + 8) * U * abs(float(scale[a])) * (xs[t].abs() @ A[a].double().abs().T)
                want[t] += v @ Bd.T
                e[t] += ((UB + (r + 8) * U) * v.abs() + (1 + UB) * e_v) @ Bd.abs().T
            assert torch.all((got[:, m:m + 1184] - want).abs() <= (1 + UB) * e + UB * want.abs())
    finally:
        del x, W, y
        torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", ["one", "mixed"])
@pytest.mark.parametrize("T", [50, 200, 600])
def test_inner_values_above_bf16s_range_stay_finite(T, kind):
    """scale (x A^T) may be any fp32 value: beyond bf16's largest, 3.39e38, its first term must not round to infinity."""
    K, M, n, r = 64, 136, 3, 8
    d, ids = _inputs(T, K, M, n, r, 70), _ids(kind, T, n, 2)
    d["x"], d["A"] = torch.zeros_like(d["x"]), torch.zeros_like(d["A"])
    d["x"][:, 5] = torch.where(torch.arange(T) % 3 == 0, -1.0, 1.0).bfloat16()
    d["A"][:, 0, 5] = 1.0                                      # x A^T = +-1 in rank 0, exactly
    d["Bm"] = (d["Bm"].float() * 2.0 ** -12).bfloat16()
    d["scale"] = torch.tensor([3.4e38, -3.3965e38, 3.4028234e38])
    y, st = _call(T, K, M, n, r, d, ids)
    assert st == 0 and torch.isfinite(y).all()
    # v exact in fp32, within 2^-16 in two bf16 terms; the sum's other terms (x W^T, zeros) are below its last bit
    want = ado.adapter_linear(_np(d["x"]), _np(d["W"]), _np(d["A"]), _np(d["Bm"]), _np(d["scale"]), ids.numpy())
    assert np.all(np.abs(_np(y) - want) <= (UB + 2.0 ** -16 + 16 * U) * np.abs(want))


@pytest.mark.parametrize("T,n,kind", [(50, 3, "mixed"), (128, 1, "one"), (129, 3, "one"), (200, 3, "mixed"), (700, 5, "runs"), (300, 40, "own")])
@pytest.mark.parametrize("r", [8, 40, 128])
def test_inner_values_keep_sixteen_bits_more_than_y(T, n, kind, r):
    """Ranks in pairs whose A rows differ in one element and whose B are each other's negative: y is the small difference
    of large terms, and inner values held in one bf16 term would miss it by 2^-9 of those."""
    K, M = 64, 200
    g = torch.Generator().manual_seed(r)
    ids = _ids(kind, T, n, 3)
    A = torch.randn(n, r // 2, K, generator=g).bfloat16()
    A2 = A.clone()
    A2[:, :, 7] = (A[:, :, 7].float() + 2.0 ** -7 * torch.randn(n, r // 2, generator=g)).bfloat16()
    b = torch.randn(n, M, r // 2, generator=g).bfloat16()
    d = dict(x=torch.randn(T, K, generator=g).bfloat16(), W=torch.zeros(M, K, dtype=bf16),
             A=torch.stack([A, A2], 2).reshape(n, r, K).contiguous(), Bm=torch.stack([b, -b], 3).reshape(n, M, r).contiguous(),
             scale=torch.tensor([(0.75, 1.0, -1.75)[i % 3] for i in range(n)]))
    y, st = _call(T, K, M, n, r, d, ids)
    assert st == 0
    x, A, Bm, sc, ids = _np(d["x"]), _np(d["A"]), _np(d["Bm"]), _np(d["scale"]), ids.numpy()
    want = ado.adapter_linear(x, _np(d["W"]), A, Bm, sc, ids)
    e = np.zeros_like(want)
    for a in range(n):
        t = np.nonzero(ids == a)[0]
        v = np.abs(sc[a] * (x[t] @ A[a].T))
        # sums of K products, then the scale; the terms, within 2^-16; sums of two terms a rank and the empty K loop's.
        # The tensor cores truncate: one addition costs up to 2 U
        e_v = 2 * (K + 8) * U * abs(sc[a]) * (np.abs(x[t]) @ np.abs(A[a]).T)
        e[t] = (e_v + (2.0 ** -16 + 2 * (2 * r + 8) * U) * (v + e_v)) @ np.abs(Bm[a]).T
    assert np.all(np.abs(_np(y) - want) <= e + UB * (np.abs(want) + e)), \
        "worst %.3g of its bound" % (np.abs(_np(y) - want) / np.maximum(e + UB * (np.abs(want) + e), 1e-30)).max()


@pytest.mark.parametrize("T,K,M,n,r,kind", [(300, 64, 136, 300, 16, "own"), (513, 128, 264, 600, 8, "own"), (700, 64, 200, 250, 32, "mixed"),
                                            (129, 64, 64, 1000, 128, "own"), (256, 72, 2816, 256, 8, "own")])
def test_blocks_of_more_adapters_than_a_word_has_bits(T, K, M, n, r, kind):
    """Up to every token of a 256-token block another adapter; some of the late slots' B hold NaN or infinities."""
    d, ids = _inputs(T, K, M, n, r, 80), _ids(kind, T, n, 9)
    clean, st = _call(T, K, M, n, r, d, ids)
    assert st == 0
    _check(d, ids, clean)
    broken = sorted({int(ids[t]) for t in (31, 32, 33, 63, 64, 100, 128, T - 1) if t < T and int(ids[t]) >= 0})
    bad = {**d, "Bm": d["Bm"].clone()}
    for k, a in enumerate(broken):
        bad["Bm"][a, M // 2 + k, r - 1] = float("nan") if k % 2 else float("inf")
    y, st = _call(T, K, M, n, r, bad, ids)
    assert st == 0
    touched = torch.zeros(T, dtype=torch.bool)
    for a in broken:
        touched |= ids == a
    same = y.cpu().view(torch.int16) == clean.cpu().view(torch.int16)
    assert same[~touched].all()
    for k, a in enumerate(broken):                             # its own rows: that column alone (sums in another order)
        t = torch.nonzero(ids == a).flatten()
        assert not torch.isfinite(y.cpu()[t][:, M // 2 + k]).any()
        cols = [m for m in range(M) if m != M // 2 + k]
        assert torch.isfinite(y.cpu()[t][:, cols]).all()
    keep = [m for m in range(M) if not M // 2 <= m < M // 2 + len(broken)]
    _check({**d, "W": d["W"][keep], "Bm": d["Bm"][:, keep]}, ids, y[:, keep].contiguous())


def test_many_token_calls_on_two_streams_and_from_graphs_that_share_a_workspace():
    """The pair kernel with its slot lists: calls that overlap have a workspace each, graphs replayed one after the other
    may share one, and nothing of an earlier replay is left in it."""
    T, K, M, n, r = 700, 256, 1032, 16, 24
    s = B.make_adapter_shape(T, K, M, n, r)
    runs = []
    for seed, kind in ((1, "mixed"), (2, "runs")):
        d, ids = _inputs(T, K, M, n, r, 90 + seed), _ids(kind, T, n, seed).cuda()
        runs.append(({k: v.cuda() for k, v in d.items()}, ids, torch.zeros(T, M, dtype=bf16, device="cuda"),
                     torch.zeros(1, dtype=i32, device="cuda"), B.new_adapter_workspace(s), torch.cuda.Stream()))

    def go(q, ws=None, stream=None):
        c, ids, y, st, own, _ = q
        B.moe_adapter_linear(s, c["x"], c["W"], c["A"], c["Bm"], c["scale"], ids, y, st, own if ws is None else ws, stream=stream)

    ref = []
    for q in runs:
        go(q)
        torch.cuda.synchronize()
        ref.append(q[2].clone())
        q[2].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for q in runs:
            go(q, stream=q[5])
    torch.cuda.synchronize()
    assert all(torch.equal(q[2], y) and int(q[3]) == 0 for q, y in zip(runs, ref))
    graphs, side = [], torch.cuda.Stream()
    for q in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            go(q, ws=runs[0][4])
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1, 0)):
        for q in runs:
            q[2].zero_()
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(q[2], y) for q, y in zip(runs, ref))
    runs[0][1].copy_(_ids("one", T, n, 1))                      # other ids in the same buffer: uniform instead of mixed
    graphs[0].replay()
    torch.cuda.synchronize()
    again = runs[0][2].clone()
    go(runs[0])
    torch.cuda.synchronize()
    assert torch.equal(again, runs[0][2]) and not torch.equal(again, ref[0])


@pytest.mark.parametrize("T,K,M,n,r", [(129, 8, 8, 1, 8), (300, 8, 16, 3, 16), (257, 16, 8, 300, 8), (1, 8, 8, 1, 128), (128, 64, 20000, 3, 128),
                                       (40, 512, 8200, 3, 24), (128, 8, 5000, 40, 64)])
@pytest.mark.parametrize("kind", ["one", "mixed"])
def test_adapter_linear_at_the_ends_of_its_ranges(T, K, M, n, r, kind):
    """The smallest widths with many tokens, the most shared memory with few, two CTAs a cluster."""
    d, ids = _inputs(T, K, M, n, r, 100), _ids(kind, T, n, T)
    y, st = _call(T, K, M, n, r, d, ids)
    assert st == 0
    _check(d, ids, y)


def _at_offset(t, elems=8):
    """The same tensor 16 bytes behind an aligned address."""
    raw = torch.empty(t.numel() + elems, dtype=t.dtype, device="cuda")
    out = raw[elems:].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("T", [3, 64, 150, 700])
def test_sixteen_byte_alignment_is_enough(T):
    K, M, n, r = 136, 264, 5, 24
    d, ids = _inputs(T, K, M, n, r, 101), _ids("mixed", T, n, 3)
    want, _ = _call(T, K, M, n, r, d, ids)
    s = B.make_adapter_shape(T, K, M, n, r)
    c = {k: _at_offset(v) if v.dtype is bf16 else v.cuda() for k, v in d.items()}
    y, st = _at_offset(torch.full((T, M), -7.0, dtype=bf16)), torch.zeros(1, dtype=i32, device="cuda")
    ws = torch.full((B.moe_adapter_workspace_bytes(s) + 16,), 255, dtype=torch.uint8, device="cuda")[16:]
    B.moe_adapter_linear(s, c["x"], c["W"], c["A"], c["Bm"], c["scale"], ids.cuda(), y, st, ws)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(y.view(torch.int16), want.view(torch.int16))
    H, I, S = 128, 64, 2
    q, shape = _shared_inputs(T, H, I, S, n, r, 102), B.make_shape(T, 128, 8, 64, 2, 1, 0)
    ref, _ = _shared_call(T, H, I, S, q, ids)
    ws = torch.full((B.moe_shared_adapted_workspace_bytes(shape, n, r) + 16,), 255, dtype=torch.uint8, device="cuda")[16:]
    y, st = _shared_call(T, H, I, S, {k: _at_offset(v) if v.dtype is bf16 else v for k, v in q.items()}, ids, ws=ws,
                         y=_at_offset(torch.zeros(T, H, dtype=bf16)))
    assert st == 0 and torch.equal(y.view(torch.int16), ref.view(torch.int16))


@pytest.mark.parametrize("T", [60, 200])
def test_adapters_beyond_four_gigabytes_of_elements(T):
    """A and B of 4.4e9 elements each, the named adapters among the last."""
    K, M, n, r = 8192, 8200, 4200, 128
    if torch.cuda.mem_get_info()[0] < 30 * 10 ** 9:
        pytest.skip("needs 20 GB")
    g = torch.Generator().manual_seed(5)
    used = torch.tensor([0, 2047, 2048, 4095, 4198, 4199])
    ids = used[torch.randint(0, len(used), (T,), generator=g)].to(i32)
    d = _inputs(T, K, M, len(used), r, 103)
    scale = torch.zeros(n)
    scale[used] = d["scale"]
    A, Bm = torch.zeros(n, r, K, dtype=bf16, device="cuda"), torch.zeros(n, M, r, dtype=bf16, device="cuda")
    A[used.cuda()], Bm[used.cuda()] = d["A"].cuda(), d["Bm"].cuda()
    try:
        y, st = _call(T, K, M, n, r, dict(x=d["x"], W=d["W"], A=A, Bm=Bm, scale=scale), ids)
    finally:
        del A, Bm
        torch.cuda.empty_cache()
    assert st == 0
    _check(d, torch.searchsorted(used, ids.long()).to(i32), y, np.arange(0, T, 7))
