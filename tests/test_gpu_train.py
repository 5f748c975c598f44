"""The calls for training the layer against their fp64 forms, at the sizes and lists where they can go wrong, in a run from the residual
to the updated weights, on side streams and from captured graphs."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as orc
from paper_2604_08133_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8          # a bf16 rounding, relative
EPS = 1e-6


def _randn(*shape, seed=0, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed * 7919 + sum(shape))
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def _np(t):
    return t.detach().double().cpu().numpy()


def _offsets(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _check_sum(got, ref, magnitude, terms, half=HALF):
    """A sum of `terms` exact products rounded once.  A tensor-core step adds 16 products and the accumulator, each cut to the largest's
    exponent: at most 17 parts of 2^-23 of the largest, which the sum of magnitudes bounds; terms / 16 steps."""
    tol = half * np.abs(ref) + (terms / 16 + 2) * 17 * 2.0 ** -23 * magnitude
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])


# ------------------------------------------------------------------------------------------------ products
LISTS = [
    # P, K, M, offsets
    (1, 8, 8, [0, 1]),
    (5, 72, 200, [0, 0, 3, 3, 4]),
    (300, 136, 264, [2, 130, 131, 131, 259]),                    # rows in front of and behind the segments, 128 and one row
    (257, 64, 512, [0, 257]),                                     # one row over a pair's tile
    (700, 200, 328, [0, 129, 256, 640]),                          # pairs: 129, 127 and 384 rows
    (1100, 320, 136, [7, 7, 7, 1100]),                            # pieces of 512 rows, odd starts
    (513, 1032, 72, [0, 1, 2, 15, 31, 48, 65, 512]),
    (40, 64, 64, list(range(0, 36)) + [36] * 30 + [40] * 3),      # 68 groups of one row, of none, of four
    (384, 96, 104, [0] + [3 * (i + 1) for i in range(128)]),      # 128 groups of three
]


@pytest.mark.parametrize("P,K,M,off", LISTS, ids=lambda v: str(v) if isinstance(v, int) else "")
def test_products(P, K, M, off):
    E = len(off) - 1
    x, dy, W, o = _randn(P, K, seed=1), _randn(P, M, seed=2), _randn(E, M, K, seed=3, std=0.1), _offsets(off)
    # what no segment holds may be anything and stays as it was
    outside = torch.ones(P, dtype=torch.bool)
    outside[off[0]:off[-1]] = False
    x[outside.cuda()], dy[outside.cuda()] = float("nan"), float("inf")
    xn, dn = np.where(outside[:, None], 0, _np(x)), np.where(outside[:, None], 0, _np(dy))
    Wn, st, s = _np(W), _status(), B.make_grouped_shape(P, K, M, E)
    y, dx = torch.full((P, M), -3.0, dtype=torch.bfloat16, device="cuda"), torch.full((P, K), -3.0, dtype=torch.bfloat16, device="cuda")
    B.moe_grouped_gemm(s, x, o, W, y, st)
    B.moe_grouped_gemm_dx(s, dy, o, W, dx, st)
    dW16, dW32 = torch.full((E, M, K), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((E, M, K), 9.0, device="cuda")
    again = torch.full((E, M, K), 0.5, device="cuda")
    B.moe_grouped_gemm_dw(s, dy, x, o, dW16, st)
    B.moe_grouped_gemm_dw(s, dy, x, o, dW32, st)
    B.moe_grouped_gemm_dw(s, dy, x, o, again, st, add=True)
    assert int(st) == 0
    assert (y[outside.cuda()] == -3).all() and (dx[outside.cuda()] == -3).all()
    inside = ~outside.numpy()
    _check_sum(_np(y)[inside], orc.product(xn, off, Wn)[inside], orc.product(abs(xn), off, abs(Wn))[inside], K)
    _check_sum(_np(dx)[inside], orc.product(dn, off, Wn, True)[inside], orc.product(abs(dn), off, abs(Wn), True)[inside], M)
    ref, mag, rows = orc.weight_gradient(dn, xn, off), orc.weight_gradient(abs(dn), abs(xn), off), max(b - a for a, b in orc.segments(off))
    _check_sum(_np(dW16), ref, mag, rows)
    _check_sum(_np(dW32), ref, mag, min(rows, 512), half=(rows // 512 + 1) * 2.0 ** -24)
    _check_sum(_np(again), ref + 0.5, mag + 0.5, min(rows, 512), half=(rows // 512 + 2) * 2.0 ** -24)


# The contraction of y or dx shared by a cluster: one row, unequal shares with an end of 8, several rounds of tiles, rows that fill no tile, an
# empty group; two, four and eight CTAs.
@pytest.mark.parametrize("P,K,M,off", [
    (1, 4096, 64, [0, 1]), (3, 72, 4104, [0, 2]), (70, 2056, 264, [0, 70]), (896, 4096, 72, np.cumsum([0] + [65, 63] * 7).tolist()),
    (500, 2048, 1000, [0, 500]), (300, 4096, 520, [5, 40, 40, 299]), (64, 4096, 4096, [0, 64])], ids=lambda v: str(v) if isinstance(v, int) else "")
def test_products_with_a_long_contraction_and_few_tiles(P, K, M, off):
    test_products(P, K, M, off)


def test_long_contractions_repeat_their_bits_on_streams_and_from_a_graph():
    P, K, M, off = 100, 2048, 2048, [0, 30, 100]
    s, o, W, x, dy, st = B.make_grouped_shape(P, K, M, 2), _offsets(off), _randn(2, M, K, seed=5), _randn(P, K), _randn(P, M, seed=1), _status()
    outs = [(torch.zeros(P, M, dtype=torch.bfloat16, device="cuda"), torch.zeros(P, K, dtype=torch.bfloat16, device="cuda")) for _ in range(4)]

    def run(out, stream=None):
        B.moe_grouped_gemm(s, x, o, W, out[0], st, stream=stream)
        B.moe_grouped_gemm_dx(s, dy, o, W, out[1], st, stream=stream)

    run(outs[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        for q, out in zip(streams, outs[1:]):
            run(out, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(outs[3])
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert int(st) == 0 and all(torch.equal(a, b) for out in outs[1:] for a, b in zip(out, outs[0]))


def test_a_groups_nan_stays_in_its_group():
    P, K, M, off = 330, 128, 192, [0, 37, 165, 165, 293]
    x, dy, W, o, st = _randn(P, K), _randn(P, M, seed=1), _randn(4, M, K, seed=2), _offsets(off), _status()
    s = B.make_grouped_shape(P, K, M, 4)

    def run():
        y, dx, dW = torch.zeros(P, M, dtype=torch.bfloat16, device="cuda"), torch.zeros(P, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, M, K, device="cuda")
        B.moe_grouped_gemm(s, x, o, W, y, st)
        B.moe_grouped_gemm_dx(s, dy, o, W, dx, st)
        B.moe_grouped_gemm_dw(s, dy, x, o, dW, st)
        return y, dx, dW

    clean = run()
    x[37:165], dy[37:165], W[1], W[2] = float("nan"), float("inf"), float("nan"), float("nan")
    y, dx, dW = run()
    for a, b in ((y, clean[0]), (dx, clean[1])):
        assert torch.equal(a[:37], b[:37]) and torch.equal(a[165:293], b[165:293]) and a[37:165].isnan().all()
    assert torch.equal(dW[0], clean[2][0]) and torch.equal(dW[3], clean[2][3]) and not dW[2].any() and dW[1].isnan().all()


def test_fp32_sums_over_many_rows_stay_near_fp32():
    """8191 rows of one sign: an accumulator that truncates would lose 2^-24 a step on average, 512 steps."""
    P, K, M = 8191, 64, 128
    x, dy = _randn(P, K).abs(), _randn(P, M, seed=1).abs()
    dW = torch.zeros(1, M, K, device="cuda")
    B.moe_grouped_gemm_dw(B.make_grouped_shape(P, K, M, 1), dy, x, _offsets([0, P]), dW, _status())
    ref = dy.double().T @ x.double()
    # 32 steps a piece, each off by at most 2^-23 of a partial sum that grows to the piece's; 16 pieces joined with one rounding each
    assert float(((dW[0].double() - ref).abs() / ref).max()) <= 32 * 2.0 ** -23 / 2 + 16 * 2.0 ** -24


@pytest.mark.parametrize("counts", [[1] * 40, [5, 3, 1, 0, 9, 2, 4, 6] * 4, [513, 1, 1, 1, 511, 15, 17, 1], [70, 0, 0, 1500, 2, 70, 0, 3]])
def test_ragged_ends_one_after_the_other(counts):
    """Many tiles a CTA, almost all with a ragged block, some with pieces: every stage of the ring takes turns between the two loaders."""
    off = np.concatenate([[0], np.cumsum(counts)]).tolist()
    P, K, M, E = off[-1], 1032, 776, len(counts)
    x, dy = _randn(P, K, seed=len(counts)), _randn(P, M, seed=3)
    out, st, s = torch.zeros(E, M, K, device="cuda"), _status(), B.make_grouped_shape(P, K, M, E)
    half = torch.zeros(E, M, K, dtype=torch.bfloat16, device="cuda")
    B.moe_grouped_gemm_dw(s, dy, x, _offsets(off), out, st)
    B.moe_grouped_gemm_dw(s, dy, x, _offsets(off), half, st)
    assert int(st) == 0
    for e, (a, b) in enumerate(orc.segments(off)):
        ref, mag = dy[a:b].double().T @ x[a:b].double(), dy[a:b].double().abs().T @ x[a:b].double().abs()
        steps = (min(b - a, 512) / 16 + 2) * 17 * 2.0 ** -23        # as in _check_sum
        assert ((out[e] - ref).abs() <= steps * mag + ((b - a) // 512 + 1) * 2.0 ** -24 * ref.abs()).all()
        assert ((half[e] - ref).abs() <= ((b - a) / 16 + 2) * 17 * 2.0 ** -23 * mag + HALF * ref.abs()).all()


@pytest.mark.parametrize("P,K,M,off", [
    (4099, 64, 64, [0, 4099]), (12153, 152, 232, [0, 10803]), (6000, 264, 136, [3, 2900, 2900, 5990]), (5000, 8, 1032, [0, 5, 5000]),
    (5000, 1032, 8, [17, 4999]), (16384, 520, 200, [0, 8000, 16384]), (9000, 72, 328, [0, 31, 63, 8999]), (2048, 1000, 1000, [1, 2048]),
    (3000, 64, 64, [0] + [100 * (i + 1) for i in range(30)])], ids=lambda v: str(v) if isinstance(v, int) else "")
def test_weight_gradients_of_long_segments_and_few_tiles(P, K, M, off):
    """The rows of a tile are shared by the CTAs of a cluster: shares of unequal length, of none, with a ragged end; NaN beside the segments."""
    E, o, st = len(off) - 1, _offsets(off), _status()
    s, x, dy = B.make_grouped_shape(P, K, M, E), _randn(P, K, seed=1), _randn(P, M, seed=2)
    for t in (x, dy):
        t[:off[0]], t[off[-1]:] = float("nan"), float("nan")
    outs = [(torch.full((E, M, K), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((E, M, K), 9.0, device="cuda"),
             torch.full((E, M, K), 0.5, device="cuda")) for _ in range(4)]

    def run(out, stream=None):
        B.moe_grouped_gemm_dw(s, dy, x, o, out[0], st, stream=stream)
        B.moe_grouped_gemm_dw(s, dy, x, o, out[1], st, stream=stream)
        B.moe_grouped_gemm_dw(s, dy, x, o, out[2], st, add=True, stream=stream)

    run(outs[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for q, out in zip(streams, outs[1:]):
        run(out, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(outs[3])
    outs[3][2].fill_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert int(st) == 0 and all(torch.equal(a, b) for out in outs[1:] for a, b in zip(out, outs[0]))
    for e, (a, b) in enumerate(orc.segments(off)):
        rows = b - a
        ref, mag = dy[a:b].double().T @ x[a:b].double(), dy[a:b].double().abs().T @ x[a:b].double().abs()
        steps = lambda n: (n / 16 + 2) * 17 * 2.0 ** -23           # as in _check_sum
        # fp32: pieces of 512 rows in each of up to 8 shares, a rounding for each and for each share
        joins = (rows / 512 + 16) * 2.0 ** -24
        assert ((outs[0][0][e].double() - ref).abs() <= (steps(rows) + joins) * mag + HALF * ref.abs()).all()
        assert ((outs[0][1][e].double() - ref).abs() <= (steps(min(rows, 512)) + joins) * mag).all()
        assert ((outs[0][2][e].double() - ref - 0.5).abs() <= (steps(min(rows, 512)) + joins) * (mag + 0.5)).all()


@pytest.mark.parametrize("P,K,M,E", [(1 << 20, 256, 128, 73), (1 << 20, 256, 256, 37), (1 << 23, 64, 64, 1)])
def test_bf16_weight_gradients_of_very_long_segments(P, K, M, E):
    """Rows of one sign: one accumulation of 2^20 rows, cut off at every step, is low by more than the result's rounding."""
    counts = [P] if E == 1 else [3, 0, 70, P - 73 - 33 - 2 * (E - 6), 33, 0] + [2] * (E - 6)
    off = np.concatenate([[0], np.cumsum(counts)]).tolist()
    g = torch.Generator(device="cuda").manual_seed(5)
    spread = 1 + torch.arange(K, device="cuda") / K            # the sums lie all over a binade
    x, dy = ((torch.rand(P, n, device="cuda", generator=g) + 0.5).mul_(f).to(torch.bfloat16) for n, f in ((K, spread), (M, 1.0)))
    dW, st, s = torch.zeros(E, M, K, dtype=torch.bfloat16, device="cuda"), _status(), B.make_grouped_shape(P, K, M, E)
    B.moe_grouped_gemm_dw(s, dy, x, _offsets(off), dW, st)
    # steps of 16 rows, each off by at most 17 parts of 2^-23 of a sum that grows evenly to its last value; then a rounding a piece: pieces of 512 rows
    # in eight shares where the one group's rows are shared, else of 32 768
    loss = (512 / 16 if E == 1 else 32768 / 16) * 17 * 2.0 ** -24 + (P / 512 / 8 + 8 if E == 1 else P / 32768) * 2.0 ** -24
    for e, (a, b) in enumerate(orc.segments(off)):
        ref = sum((dy[i:min(b, i + 131072)].double().T @ x[i:min(b, i + 131072)].double() for i in range(a, b, 131072)),
                  torch.zeros(M, K, dtype=torch.float64, device="cuda"))
        assert ((dW[e].double() - ref).abs() <= (HALF + loss) * ref).all(), (e, float(((dW[e].double() - ref) / ref).abs().max()))
    # integers: exact, so that a piece that is lost or added twice shows
    x, dy = (torch.randint(-2, 3, (P, n), device="cuda", generator=g).to(torch.bfloat16) for n in (K, M))
    again = torch.empty_like(dW)
    B.moe_grouped_gemm_dw(s, dy, x, _offsets(off), dW, st)
    B.moe_grouped_gemm_dw(s, dy, x, _offsets(off), again, st)
    for e, (a, b) in enumerate(orc.segments(off)):
        ref = sum((dy[i:min(b, i + 131072)].double().T @ x[i:min(b, i + 131072)].double() for i in range(a, b, 131072)),
                  torch.zeros(M, K, dtype=torch.float64, device="cuda"))
        assert torch.equal(dW[e], ref.float().to(torch.bfloat16)), e
    assert int(st) == 0 and torch.equal(again, dW)


@pytest.mark.parametrize("P,K,M,off", [
    (12153, 152, 232, [0, 10803]), (6000, 264, 136, [3, 2900, 2900, 5990]), (16384, 64, 64, [0, 16384]), (2048, 1000, 1000, [1, 2048]),
    (1200, 320, 776, [0, 513, 514, 515, 516, 1027, 1042, 1059, 1060, 1199]), (1642, 1032, 776, [0, 70, 70, 70, 1570, 1572, 1642])],
    ids=lambda v: str(v) if isinstance(v, int) else "")
def test_weight_gradients_of_small_integers_are_exact(P, K, M, off):
    """Products and sums of small integers are exact in fp32, so a row that is lost or taken twice shows in every type of the result."""
    E, o, st, s = len(off) - 1, _offsets(off), _status(), B.make_grouped_shape(P, K, M, len(off) - 1)
    g = torch.Generator().manual_seed(P + K)
    x, dy = (torch.randint(-3, 4, (P, n), generator=g).to(torch.bfloat16).cuda() for n in (K, M))
    half, wide = torch.empty(E, M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(E, M, K, device="cuda")
    more = torch.randint(-9, 10, (E, M, K), generator=g).float().cuda()
    added = more.clone()
    B.moe_grouped_gemm_dw(s, dy, x, o, half, st)
    B.moe_grouped_gemm_dw(s, dy, x, o, wide, st)
    B.moe_grouped_gemm_dw(s, dy, x, o, added, st, add=True)
    ref = torch.stack([dy[a:b].double().T @ x[a:b].double() for a, b in orc.segments(off)])
    assert int(st) == 0 and float(ref.abs().max()) < 2 ** 24
    assert torch.equal(wide, ref.float()) and torch.equal(half, ref.float().to(torch.bfloat16)) and torch.equal(added, more + ref.float())


def test_offsets_that_are_no_list_stay_in_bounds():
    P, K, M, E = 200, 64, 64, 5
    x, W, st, s = _randn(P, K), _randn(E, M, K, seed=1), _status(), B.make_grouped_shape(P, K, M, E)
    for off in ([0, 150, 20, 900, -5, 1 << 30], [-7, -1, 0, 0, 5, 2 ** 31 - 1], [300, 200, 100, 0, 0, 0]):
        y, dW = torch.zeros(P + 64, M, dtype=torch.bfloat16, device="cuda"), torch.zeros(E, M, K, device="cuda")
        B.moe_grouped_gemm(s, x, _offsets(off), W, y[:P], st)
        B.moe_grouped_gemm_dx(s, x, _offsets(off), W, y[:P], st)
        B.moe_grouped_gemm_dw(s, x, x, _offsets(off), dW, st)
        torch.cuda.synchronize()
        assert not y[P:].any()


def test_products_repeat_their_bits_on_side_streams_and_from_graphs():
    P, K, M, off = 900, 256, 320, [0, 300, 301, 777, 900]
    s, o, W = B.make_grouped_shape(P, K, M, 4), _offsets(off), _randn(4, M, K, seed=5)
    x, dy, st = _randn(P, K), _randn(P, M, seed=1), _status()
    outs = lambda: (torch.empty(P, M, dtype=torch.bfloat16, device="cuda"), torch.empty(P, K, dtype=torch.bfloat16, device="cuda"), torch.empty(4, M, K, device="cuda"))

    def run(o_, stream=None):
        B.moe_grouped_gemm(s, x, o, W, o_[0], st, stream=stream)
        B.moe_grouped_gemm_dx(s, dy, o, W, o_[1], st, stream=stream)
        B.moe_grouped_gemm_dw(s, dy, x, o, o_[2], st, stream=stream)

    want = outs()
    run(want)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], [outs() for _ in range(3)]
    for _ in range(5):
        for q, g in zip(streams, got):
            run(g, q)
    torch.cuda.synchronize()
    replayed = outs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(replayed)
    for t in replayed:
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for g in got + [replayed]:
        for a, b in zip(g, want):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ experts' backward pass
def _experts(T, H, N, I, K, counts, seed=0):
    off = np.concatenate([[0], np.cumsum(counts)]).tolist()
    budget = off[-1]
    g = torch.Generator().manual_seed(seed)
    tok = torch.randint(0, T, (max(budget, 1),), generator=g, dtype=torch.int32)[:budget].cuda()
    return dict(shape=B.make_shape(T, H, N, I, 0, K, 0), off=off, o=_offsets(off), budget=budget, tok=tok, x=_randn(T, H, seed=seed),
                W13=_randn(N, 2 * I, H, seed=seed + 1, std=0.1), W2=_randn(N, H, I, seed=seed + 2, std=0.1), dy=_randn(budget, H, seed=seed + 3),
                ws=None)


def _run_experts(d, x, tok, dx, dW13, dW2, st, ws=None):
    ws = B.new_ffn_backward_workspace(d["shape"], d["budget"]) if ws is None else ws
    ws.fill_(255)                                   # NaN in every 16-bit pair: nothing of a workspace is used before it is written
    B.moe_grouped_ffn_backward(d["shape"], x, tok, d["o"], d["budget"], d["W13"], d["W2"], d["dy"], dx, dW13, dW2, st, ws)


CASES = [
    (40, 128, 8, 64, 4, [1, 0, 0, 2, 0, 0, 0, 1]),
    (64, 256, 12, 192, 4, [0, 17, 3, 33, 1, 0, 64, 65, 9, 16, 15, 0]),
    (700, 192, 8, 320, 4, [129, 127, 256, 257, 0, 500, 1, 700]),     # pairs
    (600, 64, 8, 64, 8, [0, 0, 0, 0, 4800, 0, 0, 0]),
]


@pytest.mark.parametrize("T,H,N,I,K,counts", CASES, ids=["few", "ragged", "pairs", "one"])
def test_experts_backward(T, H, N, I, K, counts):
    d, st = _experts(T, H, N, I, K, counts), _status()
    dx, dW13, dW2 = torch.empty_like(d["dy"]), torch.empty_like(d["W13"]), torch.empty_like(d["W2"])
    _run_experts(d, d["x"], d["tok"], dx, dW13, dW2, st)
    assert int(st) == 0
    rows = d["x"][d["tok"].long()]
    want = orc.experts_backward(_np(rows), d["off"], _np(d["W13"]), _np(d["W2"]), _np(d["dy"]))
    for name, got, ref in zip(("dx", "dW13", "dW2"), (dx, dW13, dW2), want):
        # a factor (du or h) and the result are rounded once each, independently: sqrt(2) of one rounding's share, 2^-8 / sqrt(3) at
        # most; sums, exponentials and quotients in fp32 stay below a hundredth of it
        rms = np.sqrt(((_np(got) - ref) ** 2).mean() / (ref ** 2).mean())
        assert rms <= 1.01 * HALF * np.sqrt(2 / 3), (name, rms)
        assert not np.isnan(_np(got)).any()
        for e, n in enumerate(counts):
            if n == 0 and name != "dx":
                assert not got[e].any()
    # the rows gathered by the caller, and each output by itself: the same bits
    one = [torch.full_like(t, 7.0) for t in (dx, dW13, dW2)]
    _run_experts(d, rows.contiguous(), None, one[0], None, None, st)
    _run_experts(d, rows.contiguous(), None, None, one[1], None, st)
    _run_experts(d, d["x"], d["tok"], None, None, one[2], st)
    for a, b in zip(one, (dx, dW13, dW2)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,H,N,I,K,counts", [
    (1, 2048, 8, 320, 4, [1, 0, 1, 0, 0, 1, 0, 1]), (80, 1024, 12, 64, 12, [65, 63] * 6), (70, 1088, 8, 192, 4, [0, 17, 33, 64, 1, 65, 3, 70]),
    (14, 2048, 24, 192, 6, [3, 0, 1, 2, 5, 9] * 4), (300, 2048, 8, 128, 4, [0, 300, 0, 17, 0, 0, 0, 0])], ids=["token", "rounds", "unequal", "two", "skewed"])
def test_experts_backward_of_few_tiles(T, H, N, I, K, counts):
    """Clusters of eight, four and two CTAs share the contraction of a tile: one round and several, shares of unequal length."""
    test_experts_backward(T, H, N, I, K, counts)


@pytest.mark.parametrize("T,H,I,S", [(1, 2048, 128, 3), (70, 1088, 64, 2)])
def test_shared_experts_backward_of_few_tiles(T, H, I, S):
    test_shared_experts_backward(T, H, I, S)


@pytest.mark.parametrize("T,H,I,S", [(1, 64, 64, 1), (37, 192, 128, 2), (300, 256, 192, 3), (64, 128, 320, 1), (65, 128, 64, 4)])
def test_shared_experts_backward(T, H, I, S):
    s, st = B.make_shape(T, H, 8, I, S, 1, 0), _status()
    x, W13, W2, dy = _randn(T, H), _randn(S, 2 * I, H, seed=1, std=0.1), _randn(S, H, I, seed=2, std=0.1), _randn(T, H, seed=3)
    ws = B.new_shared_ffn_backward_workspace(s)
    ws.fill_(255)
    dx, dW13, dW2 = torch.empty_like(x), torch.empty_like(W13), torch.empty_like(W2)
    B.moe_shared_ffn_backward(s, x, W13, W2, dy, dx, dW13, dW2, st, ws)
    assert int(st) == 0
    each = [orc.experts_backward(_np(x), [0, T], _np(W13[k:k + 1]), _np(W2[k:k + 1]), _np(dy)) for k in range(S)]
    for got, ref in ((dx, sum(e[0] for e in each)), (dW13, np.concatenate([e[1] for e in each])), (dW2, np.concatenate([e[2] for e in each]))):
        assert np.sqrt(((_np(got) - ref) ** 2).mean() / (ref ** 2).mean()) <= 1.01 * HALF * np.sqrt(2 / 3)      # as for the routed experts
    one = [torch.full_like(t, 7.0) for t in (dx, dW13, dW2)]
    for k in range(3):
        B.moe_shared_ffn_backward(s, x, W13, W2, dy, *[o if j == k else None for j, o in enumerate(one)], st, ws)
        assert torch.equal(one[k], (dx, dW13, dW2)[k])


@pytest.mark.parametrize("T,H,I,S", [(33000, 64, 64, 2), (70001, 128, 64, 1)])
def test_shared_experts_backward_of_many_tokens(T, H, I, S):
    """Segments beyond the 32 768 rows of one accumulation, two products a launch."""
    test_shared_experts_backward(T, H, I, S)


def test_experts_backward_of_nothing():
    d, st = _experts(10, 64, 8, 64, 2, [0] * 8), _status()
    dW13, dW2 = torch.ones_like(d["W13"]), torch.ones_like(d["W2"])
    ws = B.new_ffn_backward_workspace(d["shape"], 0)
    B.moe_grouped_ffn_backward(d["shape"], None, None, d["o"], 0, d["W13"], d["W2"], None, None, dW13, dW2, st, ws)
    assert int(st) == 0 and not dW13.any() and not dW2.any()


def test_experts_backward_leaves_rows_of_no_segment():
    d, st = _experts(50, 128, 8, 64, 4, [3, 0, 40, 0, 0, 1, 0, 100]), _status()
    d["o"] = _offsets([min(v, 90) for v in d["off"]])          # the last 54 rows belong to nobody
    d["dy"][90:] = float("nan")
    dx, dW13, dW2 = torch.full_like(d["dy"], -3.0), torch.empty_like(d["W13"]), torch.empty_like(d["W2"])
    _run_experts(d, d["x"], d["tok"], dx, dW13, dW2, st)
    assert (dx[90:] == -3).all() and not dW13.isnan().any() and not dW2.isnan().any() and not dx[:90].isnan().any()


def test_experts_with_saturated_gates_stay_finite():
    d, st = _experts(64, 64, 8, 64, 2, [16] * 8), _status()
    d["W13"][:, :64] *= 100.0                                   # u1 far beyond where exp overflows in fp32
    dx, dW13, dW2 = torch.empty_like(d["dy"]), torch.empty_like(d["W13"]), torch.empty_like(d["W2"])
    _run_experts(d, d["x"], d["tok"], dx, dW13, dW2, st)
    with np.errstate(over="ignore"):
        want = orc.experts_backward(_np(d["x"][d["tok"].long()]), d["off"], _np(d["W13"]), _np(d["W2"]), _np(d["dy"]))
    for got, ref in zip((dx, dW13, dW2), want):
        assert np.isfinite(_np(got)).all()
        assert np.sqrt(((_np(got) - ref) ** 2).mean() / (ref ** 2).mean()) <= 1.01 * HALF * np.sqrt(2 / 3)


def test_experts_backward_on_three_streams_and_from_two_graphs():
    """The launches of a call overlap one another; calls on other streams, and graphs that share a workspace, must not see it."""
    cases = [_experts(90, 192, 8, 128, 4, [17, 0, 3, 33, 1, 64, 65, 9], seed=k) for k in range(2)]
    cases.append(_experts(600, 192, 8, 128, 4, [129, 127, 256, 257, 0, 500, 1, 700], seed=7))      # pairs
    outs = lambda d: (torch.zeros_like(d["dy"]), torch.zeros_like(d["W13"]), torch.zeros_like(d["W2"]))
    st, ws = _status(), [B.new_ffn_backward_workspace(d["shape"], d["budget"]) for d in cases]

    def run(d, o, w, stream=None):
        B.moe_grouped_ffn_backward(d["shape"], d["x"], d["tok"], d["o"], d["budget"], d["W13"], d["W2"], d["dy"], *o, st, w, stream=stream)

    want = [outs(d) for d in cases]
    for d, o, w in zip(cases, want, ws):
        run(d, o, w)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [outs(d) for d in cases]
    for _ in range(10):
        for d, o, w, q in zip(cases, got, ws, streams):
            run(d, o, w, q)
    torch.cuda.synchronize()
    big = max(ws, key=torch.numel)
    replayed, graphs = [outs(d) for d in cases], []
    for d, o in zip(cases, replayed):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(d, o, big)                       # one workspace for all of them, one after the other
            run(d, o, big)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert int(st) == 0
    for w_, a, b in zip(want, got, replayed):
        for x, y, z in zip(w_, a, b):
            assert torch.equal(x, y) and torch.equal(x, z)


def test_results_are_complete_for_whoever_waits_for_the_call():
    """The last launch may start before the one ahead of it has ended; what follows the call, on its stream or behind an event, sees all outputs."""
    d, st = _experts(64, 512, 8, 256, 4, [9, 30, 0, 64, 1, 50, 77, 5]), _status()
    ws, side = B.new_ffn_backward_workspace(d["shape"], d["budget"]), torch.cuda.Stream()
    dx, dW13, dW2 = torch.empty_like(d["dy"]), torch.empty_like(d["W13"]), torch.empty_like(d["W2"])
    first = None
    for _ in range(20):
        for t in (dx, dW13, dW2):
            t.fill_(float("nan"))
        B.moe_grouped_ffn_backward(d["shape"], d["x"], d["tok"], d["o"], d["budget"], d["W13"], d["W2"], d["dy"], dx, dW13, dW2, st, ws)
        e = torch.cuda.Event()
        e.record()
        side.wait_event(e)
        with torch.cuda.stream(side):
            seen = [t.clone() for t in (dx, dW13, dW2)]
        torch.cuda.current_stream().wait_stream(side)
        first = first or seen
        for a, b in zip(seen, first):
            assert torch.equal(a, b) and not a.isnan().any()


# ------------------------------------------------------------------------------------------------ norms
def _norm_inputs(T, H, G, seed=0):
    return dict(r=_randn(T, H, seed=seed), y=_randn(T, H, seed=seed + 1, std=0.3), gate=_randn(T, G, seed=seed + 2) if G else None,
                wp=1 + 0.2 * _randn(H, seed=seed + 3, dtype=torch.float32), wn=1 + 0.2 * _randn(H, seed=seed + 4, dtype=torch.float32),
                scale=torch.full((1,), -0.7, device="cuda"), dn=_randn(T, H, seed=seed + 5), dr=_randn(T, H, seed=seed + 6))


def _opt(t):
    return None if t is None else _np(t)


@pytest.mark.parametrize("T,H,G,as_is", [(1, 8, 0, False), (3, 8, 8, False), (1, 2048, 1, False), (130, 264, 1, True), (77, 1000, 1000, False),
                                         (9, 4096, 4096, False), (5, 4104, 1, False), (301, 8192, 0, True), (4, 8184, 8184, False), (2500, 64, 1, False)])
def test_block_norm_and_its_gradients(T, H, G, as_is):
    d, s = _norm_inputs(T, H, G), B.make_norm_shape(T, H, G, EPS, as_is)
    ro, no = torch.empty_like(d["r"]), torch.empty_like(d["r"])
    B.moe_block_norm(s, d["r"], d["y"], d["wp"], d["gate"], d["scale"], d["wn"], ro, no)
    want = orc.norm_r(_np(d["r"]), _np(d["y"]), _np(d["wp"]), _opt(d["gate"]), -0.7, EPS, as_is)
    size = np.abs(_np(d["r"])) + np.abs(want - _np(d["r"]))
    # one rounding to bf16; in fp32 a handful of roundings, a sum of H squares in pieces, an exponential and a quotient: 32 parts of 2^-24
    assert (np.abs(_np(ro) - want) <= HALF * np.abs(want) + 32 * 2.0 ** -24 * size).all()
    want = orc.norm_n(_np(ro), _np(d["wn"]), EPS)
    assert (np.abs(_np(no) - want) <= (HALF + 32 * 2.0 ** -24) * np.abs(want)).all()

    ws = B.new_norm_workspace(s)
    ws.fill_(255)
    out = dict(d_r=torch.empty_like(ro), d_y=torch.empty_like(ro), d_gate=None if not G else torch.empty_like(d["gate"]),
               dw_post=torch.empty(H, device="cuda"), dw_pre=torch.empty(H, device="cuda"), d_scale=torch.empty(1, device="cuda"))
    B.moe_block_norm_backward(s, ro, d["y"], d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], d["dr"], *out.values(), ws)
    want = orc.norm_backward(_np(ro), _np(d["y"]), _np(d["wp"]), _opt(d["gate"]), -0.7, _np(d["wn"]), _np(d["dn"]), _np(d["dr"]), EPS, as_is)
    for name, got in out.items():
        if got is None:
            continue
        half = HALF if got.dtype is torch.bfloat16 else 2.0 ** -24
        # the terms carry the roundings above twice over; sums over rows add one more part each for at most T / (CTAs) + 16 of them
        slack = (64 + (16 + T / 148 if name.startswith("dw") else 0)) * 2.0 ** -24
        bad = ~(np.abs(_np(got) - want[name]) <= half * np.abs(want[name]) + slack * want["|" + name + "|"])
        assert not bad.any(), (name, np.abs(_np(got) - want[name]).max(), int(bad.sum()))
    # the same bits again, and each output by itself
    for name, got in out.items():
        if got is None:
            continue
        alone = {k: torch.full_like(v, 5.0) if k == name else None for k, v in out.items()}
        B.moe_block_norm_backward(s, ro, d["y"], d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], d["dr"], *alone.values(), ws)
        assert torch.equal(alone[name], got), name


# rows that a CTA takes at a time: 1, 2, 3, 8, 15, two and four of wide rows, uneven last ones, pieces that a thread does not have
@pytest.mark.parametrize("T,H,G", [(148, 256, 1), (149, 256, 256), (2221, 256, 0), (445, 1016, 1), (1333, 1024, 1024), (2300, 512, 1),
                                   (1500, 2048, 1), (593, 2040, 2040), (297, 4096, 4096), (300, 4104, 1), (150, 5120, 0)])
def test_gradients_of_rows_that_share_a_cta(T, H, G):
    test_block_norm_and_its_gradients(T, H, G, False)


def test_norm_gradients_without_d_n_at_the_smallest_eps():
    T, H = 200, 1000
    d = _norm_inputs(T, H, 1)
    d["y"][3] = 0
    s = B.make_norm_shape(T, H, 1, 1e-38)
    dr, dy, dg, ws = torch.empty_like(d["r"]), torch.empty_like(d["r"]), torch.empty_like(d["gate"]), B.new_norm_workspace(s)
    dw, ds = torch.empty(H, device="cuda"), torch.empty(1, device="cuda")
    B.moe_block_norm_backward(s, None, d["y"], d["wp"], d["gate"], d["scale"], None, None, d["dr"], dr, dy, dg, dw, None, ds, ws)
    assert torch.equal(dr, d["dr"])
    # y of zeros: rms is sqrt(eps), its gradient the only one beyond bf16's range or close to it
    assert all(torch.isfinite(o).all() for o in (dg, dw, ds)) and not torch.isnan(dy).any()
    want = orc.norm_backward(_np(d["r"]), _np(d["y"]), _np(d["wp"]), _np(d["gate"]), -0.7, _np(d["wn"]), np.zeros((T, H)), _np(d["dr"]), 1e-38, False)
    ok = [t for t in range(T) if t != 3]
    slack = 64 * 2.0 ** -24             # as above
    assert (np.abs(_np(dy) - want["d_y"])[ok] <= HALF * np.abs(want["d_y"])[ok] + slack * want["|d_y|"][ok]).all()
    assert (np.abs(_np(dg) - want["d_gate"]) <= HALF * np.abs(want["d_gate"]) + slack * want["|d_gate|"]).all()


@pytest.mark.parametrize("G", [0, 1, 1000])
@pytest.mark.parametrize("eps,r_sizes,y_sizes", [(1e-30, [0.0, 1e-15, 1.0, 1e15, 1e17], [0.0, 1e-15, 1.0, 1e15]), (1e-45, [0.0, 1.0], [1.0]),
                                                 (1e-45, [1.0], [0.0, 1.0]), (1e-6, [0.0, 1e-15, 1e15, 1e17], [0.0, 1e15, 1e17])])
def test_norm_gradients_at_the_ends_of_fp32(eps, r_sizes, y_sizes, G):
    """Rows whose root mean square, or eps, is so far from one that its cube leaves fp32 while the gradients do not."""
    T, H = 160, 1000
    d, s, eps = _norm_inputs(T, H, G), B.make_norm_shape(T, H, G, eps), float(np.float32(eps))
    size = lambda sizes, every: torch.tensor([sizes[t // every % len(sizes)] for t in range(T)], device="cuda")[:, None]
    r = (d["r"].float() * size(r_sizes, 1)).to(torch.bfloat16)
    y = (d["y"].float() * size(y_sizes, len(r_sizes))).to(torch.bfloat16)
    for dr_out in (d["dr"], None):
        ws = B.new_norm_workspace(s)
        out = dict(d_r=torch.empty_like(r), d_y=torch.empty_like(r), d_gate=None if not G else torch.empty_like(d["gate"]),
                   dw_post=torch.empty(H, device="cuda"), dw_pre=torch.empty(H, device="cuda"), d_scale=torch.empty(1, device="cuda"))
        B.moe_block_norm_backward(s, r, y, d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], dr_out, *out.values(), ws)
        want = orc.norm_backward(_np(r), _np(y), _np(d["wp"]), _opt(d["gate"]), -0.7, _np(d["wn"]), _np(d["dn"]),
                                 np.zeros((T, H)) if dr_out is None else _np(dr_out), eps)
        for name, got in out.items():
            if got is None:
                continue
            assert torch.isfinite(got).all(), name
            # bounds as in test_block_norm_and_its_gradients
            half = HALF if got.dtype is torch.bfloat16 else 2.0 ** -24
            slack = (64 + (16 + T / 148 if name.startswith("dw") else 0)) * 2.0 ** -24
            bad = ~(np.abs(_np(got) - want[name]) <= half * np.abs(want[name]) + slack * want["|" + name + "|"])
            assert not bad.any(), (name, np.argwhere(bad)[:4], _np(got)[bad][:4], want[name][bad][:4])


@pytest.mark.parametrize("G", [1, 1000])
def test_gradients_of_gates_that_are_almost_open(G):
    """sigmoid' keeps its relative accuracy where sigmoid is one but for a few units of fp32, or one exactly."""
    T, H = 150, 1000
    d, s = _norm_inputs(T, H, G), B.make_norm_shape(T, H, G, EPS)
    at = torch.tensor([-20.0, -12.0, -8.0, 8.0, 12.0, 16.0, 17.0, 20.0], device="cuda")
    d["gate"] = at[torch.arange(T * G, device="cuda") % 8].reshape(T, G).to(torch.bfloat16)
    dg = torch.empty_like(d["gate"])
    B.moe_block_norm_backward(s, d["r"], d["y"], d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], d["dr"], None, None, dg, None, None, None)
    want = orc.norm_backward(_np(d["r"]), _np(d["y"]), _np(d["wp"]), _np(d["gate"]), -0.7, _np(d["wn"]), _np(d["dn"]), _np(d["dr"]), EPS)
    # as in test_block_norm_and_its_gradients, and an exponential of 20: 2 + 1.173 * 20 units of 2^-23
    slack = (64 + 2 * 26) * 2.0 ** -24
    assert (np.abs(_np(dg) - want["d_gate"]) <= HALF * np.abs(want["d_gate"]) + slack * want["|d_gate|"]).all()
    # far out: shut and open to the same side of zero as the oracle's at 20, finite, and symmetric in the gate
    far = {}
    for g in (60.0, -60.0):
        d["gate"] = torch.full_like(d["gate"], g)
        B.moe_block_norm_backward(s, d["r"], d["y"], d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], d["dr"], None, None, dg, None, None, None)
        far[g] = _np(dg)
    # the same products times exp(-60) / (1 + exp(-60))^2 on either side: a rounding each, and two exponentials of 60
    assert (np.abs(far[60.0] - far[-60.0]) <= (2 * HALF + 4 * 73 * 2.0 ** -23) * np.abs(far[60.0])).all() and np.abs(far[60.0]).max() > 0


@pytest.mark.parametrize("T,H", [(5, 64), (600, 2048)])
def test_block_norm_without_its_options(T, H):
    d, s = _norm_inputs(T, H, 0), B.make_norm_shape(T, H)
    ones = torch.ones(H, device="cuda")
    one = torch.ones(1, device="cuda")
    a, b, c, e = (torch.empty_like(d["r"]) for _ in range(4))
    B.moe_block_norm(s, d["r"], d["y"], None, None, None, None, a, b)
    B.moe_block_norm(s, d["r"], d["y"], ones, None, one, ones, c, e)
    assert torch.equal(a, c) and torch.equal(b, e)
    B.moe_block_norm(s, d["r"], d["y"], None, None, None, None, c, None)                 # behind the last block
    assert torch.equal(a, c)
    B.moe_block_norm(s, a, None, None, None, None, d["wn"], None, c)                      # in front of the first
    want = orc.norm_n(_np(a), _np(d["wn"]), EPS)
    assert (np.abs(_np(c) - want) <= (HALF + 32 * 2.0 ** -24) * np.abs(want)).all()
    # in place: r_out over r, n_out over y
    r, y = d["r"].clone(), d["y"].clone()
    B.moe_block_norm(s, r, y, None, None, None, None, r, y)
    assert torch.equal(r, a) and torch.equal(y, b)
    # gradients with one of the two sources, and through the norm alone
    dr = torch.empty_like(a)
    B.moe_block_norm_backward(s, None, d["y"], None, None, None, None, None, d["dr"], dr, None, None, None, None, None)
    assert torch.equal(dr, d["dr"])
    zero = torch.zeros_like(a)
    got, want = torch.empty_like(a), torch.empty_like(a)
    B.moe_block_norm_backward(s, a, d["y"], None, None, None, d["wn"], d["dn"], None, got, None, None, None, None, None)
    B.moe_block_norm_backward(s, a, d["y"], None, None, None, d["wn"], d["dn"], zero, want, None, None, None, None, None)
    assert torch.equal(got, want)
    ws, dw = B.new_norm_workspace(s), torch.empty(H, device="cuda")
    B.moe_block_norm_backward(s, a, None, None, None, None, d["wn"], d["dn"], None, got, None, None, None, dw, None, ws)
    assert torch.equal(got, want)
    # d_r over d_n, d_y over y
    dn, y = d["dn"].clone(), d["y"].clone()
    dy = torch.empty_like(y)
    B.moe_block_norm_backward(s, a, d["y"], None, None, None, d["wn"], d["dn"], d["dr"], want, dy, None, None, None, None)
    B.moe_block_norm_backward(s, a, y, None, None, None, d["wn"], dn, d["dr"], dn, y, None, None, None, None)
    assert torch.equal(dn, want) and torch.equal(y, dy)


def test_a_norms_row_depends_on_itself_alone():
    T, H = 300, 192
    d, s = _norm_inputs(T, H, H), B.make_norm_shape(T, H, H)

    def run():
        ro, no, dr, dy, dg = (torch.empty_like(d["r"]) for _ in range(5))
        B.moe_block_norm(s, d["r"], d["y"], d["wp"], d["gate"], d["scale"], d["wn"], ro, no)
        B.moe_block_norm_backward(s, ro, d["y"], d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], d["dr"], dr, dy, dg, None, None, None)
        return ro, no, dr, dy, dg

    clean = run()
    d["r"][7], d["y"][8], d["gate"][9], d["dn"][10] = float("nan"), float("inf"), float("nan"), float("inf")
    d["gate"][20], d["gate"][21] = float("inf"), float("-inf")               # open and shut: no NaN
    keep = [i for i in range(T) if i not in (7, 8, 9, 10, 20, 21)]
    for a, b in zip(run(), clean):
        assert torch.equal(a[keep], b[keep]) and torch.isfinite(a[20:22]).all()


def test_block_norm_on_streams_and_from_a_graph():
    T, H = 500, 1000
    d, s = _norm_inputs(T, H, H), B.make_norm_shape(T, H, H)
    sets = [dict(ro=torch.empty_like(d["r"]), no=torch.empty_like(d["r"]), dr=torch.empty_like(d["r"]), dy=torch.empty_like(d["r"]),
                 dg=torch.empty_like(d["gate"]), dp=torch.empty(H, device="cuda"), dq=torch.empty(H, device="cuda"), ds=torch.empty(1, device="cuda"),
                 ws=B.new_norm_workspace(s)) for _ in range(4)]

    def run(o, stream=None):
        B.moe_block_norm(s, d["r"], d["y"], d["wp"], d["gate"], d["scale"], d["wn"], o["ro"], o["no"], stream=stream)
        B.moe_block_norm_backward(s, o["ro"], d["y"], d["wp"], d["gate"], d["scale"], d["wn"], d["dn"], d["dr"], o["dr"], o["dy"], o["dg"],
                                  o["dp"], o["dq"], o["ds"], o["ws"], stream=stream)

    run(sets[0])
    torch.cuda.synchronize()
    for _ in range(5):
        for o, q in zip(sets[1:3], (torch.cuda.Stream(), torch.cuda.Stream())):
            run(o, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(sets[3])
    graph.replay()
    torch.cuda.synchronize()
    for o in sets[1:]:
        for k in ("ro", "no", "dr", "dy", "dg", "dp", "dq", "ds"):
            assert torch.equal(o[k], sets[0][k]), k


def test_zero_rows_have_finite_norms():
    d, s = _norm_inputs(4, 256, 0), B.make_norm_shape(4, 256)
    d["r"].zero_(), d["y"].zero_()
    ro, no, dr, dy = (torch.empty_like(d["r"]) for _ in range(4))
    B.moe_block_norm(s, d["r"], d["y"], d["wp"], None, d["scale"], d["wn"], ro, no)
    B.moe_block_norm_backward(s, ro, d["y"], d["wp"], None, d["scale"], d["wn"], d["dn"], d["dr"], dr, dy, None, None, None, None)
    assert not ro.any() and not no.any() and torch.isfinite(dr).all() and torch.isfinite(dy).all()


# ------------------------------------------------------------------------------------------------ AdamW
BETA1, BETA2, AEPS = 0.9, 0.999, 1e-8


def _hyper(step, lr=1e-2, clip=0.5):
    return torch.tensor([lr, 1 - BETA1 ** step, 1 - BETA2 ** step, clip], device="cuda")


def _entries(sizes, eight, bf16, grad16, copy=True, seed=0):
    items = []
    for k, n in enumerate(sizes):
        it = dict(param=_randn(n, seed=seed + 9 * k, dtype=torch.bfloat16 if bf16 else torch.float32), weight_decay=0.1 * (k % 3),
                  grad=_randn(n, seed=seed + 9 * k + 1, std=0.01, dtype=torch.bfloat16 if grad16 else torch.float32))
        if eight:
            blocks = -(-n // 256)
            it.update(m=torch.zeros(n, dtype=torch.uint8, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                      m_scale=torch.zeros(blocks, device="cuda"), v_scale=torch.zeros(blocks, device="cuda"))
        else:
            it.update(m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
        if copy and k % 2 == 0:
            it["copy"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        items.append(it)
    return items


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("bf16,grad16", [(False, False), (False, True), (True, True), (True, False)])
def test_adamw_steps(eight, bf16, grad16):
    sizes = [1, 255, 256, 257, 4096, 4097, 10001, 8]
    items, st = _entries(sizes, eight, bf16, grad16), _status()
    tensors = B.make_adamw_tensors(items)
    p_ref = [_np(it["param"]) for it in items]
    m_ref, v_ref = [np.zeros(n, np.float32) for n in sizes], [np.zeros(n, np.float32) for n in sizes]
    for step in range(1, 4):
        for k, it in enumerate(items):
            it["grad"].copy_(_randn(sizes[k], seed=100 * step + k, std=0.01, dtype=it["grad"].dtype))
            if sizes[k] > 300:
                it["grad"][5:280] = 0                            # some never move, as rows of no token
        h = _hyper(step)
        B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, h, st)
        lr, b1, b2, clip = _np(h)
        for k, it in enumerate(items):
            g = it["grad"].float().cpu().numpy()
            p64, _, _ = orc.adamw(p_ref[k], g.astype(np.float64), m_ref[k].astype(np.float64), v_ref[k].astype(np.float64), lr, b1, b2, clip, BETA1,
                                  BETA2, AEPS, it["weight_decay"])
            got = _np(it["param"])
            # parameter and step: four fp32 roundings each, the moments' three, a root, a quotient of two units: 16 parts of 2^-24
            tol = 16 * 2.0 ** -24 * (np.abs(p_ref[k]) + np.abs(p64 - p_ref[k])) + (HALF * np.abs(p64) if bf16 else 0)
            assert (np.abs(got - p64) <= tol).all()
            if "copy" in it:
                assert torch.equal(it["copy"], it["param"].to(torch.bfloat16))
            m, v = orc.moments_fp32(g, m_ref[k], v_ref[k], clip, BETA1, BETA2)
            if eight:
                for name, codes, values in (("m", orc.m_codes, orc.m_values), ("v", orc.v_codes, orc.v_values)):
                    c, s = codes(m if name == "m" else v)
                    assert np.array_equal(it[name].cpu().numpy(), c), name
                    assert np.array_equal(it[name + "_scale"].cpu().numpy(), s), name
                    if name == "m":
                        m_ref[k] = values(c, s)
                    else:
                        v_ref[k] = values(c, s)
            else:
                assert np.array_equal(it["m"].cpu().numpy(), m) and np.array_equal(it["v"].cpu().numpy(), v)
                m_ref[k], v_ref[k] = m, v
            p_ref[k] = got
    assert int(st) == 0
    if eight:
        m32, v32 = [torch.empty(n, device="cuda") for n in sizes], [torch.empty(n, device="cuda") for n in sizes]
        B.moe_adamw_states_read(tensors, m32, v32)
        for k in range(len(sizes)):
            assert np.array_equal(m32[k].cpu().numpy(), m_ref[k]) and np.array_equal(v32[k].cpu().numpy(), v_ref[k])
        before = [(it["m"].clone(), it["v"].clone()) for it in items]
        for it in items:
            it["m"].fill_(77), it["v"].fill_(77)
        B.moe_adamw_states_write(tensors, m32, v32, st)
        # the block's largest value is held exactly but for roundings, so writing what was read gives the same codes
        for it, (m, v) in zip(items, before):
            assert torch.equal(it["m"] & 127, m & 127) and torch.equal(it["v"], v)
        assert int(st) == 0


@pytest.mark.parametrize("count", [8, 9, 65, 401])
def test_adamw_lists_of_any_length(count):
    sizes = [1 + 37 * k % 700 for k in range(count)]
    items, st = _entries(sizes, False, False, False, copy=False), _status()
    before = [it["param"].clone() for it in items]
    B.moe_adamw_step(B.make_adamw_tensors(items), BETA1, BETA2, AEPS, _hyper(1), st)
    for it, p in zip(items, before):
        want = orc.adamw(_np(p), _np(it["grad"]), 0.0, 0.0, *_np(_hyper(1)), BETA1, BETA2, AEPS, it["weight_decay"])[0]
        assert (np.abs(_np(it["param"]) - want) <= 16 * 2.0 ** -24 * (np.abs(_np(p)) + np.abs(want - _np(p)))).all()
    assert int(st) == 0


def test_adamw_reports_what_is_not_finite_and_touches_nothing_else():
    for eight in (False, True):
        items = _entries([300, 5000], eight, False, False)
        guard = [it["param"].clone() for it in items]
        tensors, st = B.make_adamw_tensors(items), _status()
        B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, _hyper(1, lr=0.0), st)
        assert int(st) == 0 and all(torch.equal(it["param"], g) for it, g in zip(items, guard))
        items[1]["grad"][4999] = float("inf")
        B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, _hyper(2), st)
        assert int(st) == 1 << B.MOE_ERR_NONFINITE
        assert torch.isfinite(items[0]["param"]).all() and torch.isfinite(items[1]["param"][:4999]).all()
    m, v = [torch.zeros(300, device="cuda"), torch.zeros(5000, device="cuda")], [torch.zeros(300, device="cuda"), torch.zeros(5000, device="cuda")]
    for bad in (float("nan"), -1.0):
        v[0][7] = bad
        st = _status()
        B.moe_adamw_states_write(tensors, m, v, st)
        assert int(st) == 1 << B.MOE_ERR_NONFINITE


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("grad16", [False, True])
def test_adamw_reports_a_second_moment_that_overflows(eight, grad16):
    """A finite gradient whose square is beyond fp32: reported in the step that meets it, and the values beside it stay finite."""
    items = _entries([300, 5000], eight, False, grad16)
    tensors, st = B.make_adamw_tensors(items), _status()
    B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, _hyper(1), st)
    assert int(st) == 0
    items[1]["grad"][2100] = 1e22
    before = items[1]["param"].clone()
    B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, _hyper(2), st)
    assert int(st) == 1 << B.MOE_ERR_NONFINITE
    # a step of AdamW is at most lr / sqrt(1 - beta2) for each element, whatever the gradients
    for step in (3, 4):
        items[1]["grad"][2100] = 0.01
        for it in items:
            assert torch.isfinite(it["param"]).all()
            if eight:
                assert torch.isfinite(it["m_scale"]).all() and torch.isfinite(it["v_scale"]).all()
        B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, _hyper(step), st)
    assert all(torch.isfinite(it["param"]).all() for it in items)
    assert float((items[1]["param"] - before).abs().max()) <= 3 * 1e-2 / np.sqrt(1 - BETA2) + 0.1
    if eight:
        m32, v32 = [[torch.empty(n, device="cuda") for n in (300, 5000)] for _ in range(2)]
        B.moe_adamw_states_read(tensors, m32, v32)
        assert all(torch.isfinite(t).all() for t in m32 + v32)
        assert float(v32[1][2100]) > 1e38 and float(v32[1].max()) == float(v32[1][2100])
        st.zero_()
        v32[1][2100] = float("inf")                      # written from outside: reported as well, the block's scale finite
        B.moe_adamw_states_write(tensors, m32, v32, st)
        assert int(st) == 1 << B.MOE_ERR_NONFINITE and torch.isfinite(items[1]["v_scale"]).all()
        st.zero_()
        B.moe_adamw_step(tensors, BETA1, BETA2, AEPS, _hyper(5), st)
        assert int(st) == 0


def test_adamw_states_written_from_any_moments():
    sizes = [1, 255, 256, 257, 4097, 10001]
    items, st = _entries(sizes, True, False, False), _status()
    for it in items:
        it["m"].fill_(99), it["v"].fill_(99), it["m_scale"].fill_(5.0), it["v_scale"].fill_(5.0)
    spread = [torch.exp(4 * _randn(n, seed=70 + k, dtype=torch.float32)) for k, n in enumerate(sizes)]
    m32 = [1e-3 * _randn(n, seed=40 + k, dtype=torch.float32) * f for k, (n, f) in enumerate(zip(sizes, spread))]
    v32 = [(1e-3 * _randn(n, seed=50 + k, dtype=torch.float32) * f).square() for k, (n, f) in enumerate(zip(sizes, spread))]
    m32[4][256:512], v32[4][512:768], m32[5][300], v32[5][301] = 0.0, 0.0, -0.0, -0.0
    m32[5][1024:1280] *= 1e-30                       # a block below 2^-100
    B.moe_adamw_states_write(B.make_adamw_tensors(items), m32, v32, st)
    assert int(st) == 0
    for it, m, v in zip(items, m32, v32):
        for name, (codes, scales) in (("m", orc.m_codes(m.cpu().numpy())), ("v", orc.v_codes(v.cpu().numpy()))):
            assert np.array_equal(it[name].cpu().numpy(), codes), name
            assert np.array_equal(it[name + "_scale"].cpu().numpy(), scales), name


def test_adamw_from_a_graph_takes_new_hyper_values():
    def fresh():
        return _entries([1000, 70000], True, False, True)
    a, b, st = fresh(), fresh(), _status()
    ta, tb, h = B.make_adamw_tensors(a), B.make_adamw_tensors(b), _hyper(1)
    for step in (1, 2, 3):
        B.moe_adamw_step(ta, BETA1, BETA2, AEPS, _hyper(step, lr=0.01 / step), st)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        B.moe_adamw_step(tb, BETA1, BETA2, AEPS, h, st, stream=side)
    for step in (1, 2, 3):
        h.copy_(_hyper(step, lr=0.01 / step))
        graph.replay()
        torch.cuda.synchronize()
    for x, y in zip(a, b):
        for k in x:
            assert torch.equal(x[k], y[k]) if torch.is_tensor(x[k]) else x[k] == y[k], k


def test_the_list_of_tensors_refuses():
    def one(**kw):
        it = _entries([300], True, False, True)[0]
        it["copy"] = None
        it.update(kw)
        return it
    f = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt, device="cuda")
    shared = f(600)
    for items in ([one(param=f(300, torch.float16))], [one(grad=f(299))], [one(m=f(300))], [one(v=f(300))], [one(m_scale=f(1))], [one(v_scale=None)],
                  [one(copy=f(300))], [one(param=f(600)[::2])], [one(grad=torch.zeros(300))], [one(), None], [one(param=shared[:300]), one(param=shared[100:400])],
                  [one(param=shared[:300]), one(grad=shared[100:400])]):
        with pytest.raises(B.MoeError) as e:
            B.make_adamw_tensors(items)
        assert e.value.status == B.MOE_ERR_ARG
    B.make_adamw_tensors([one(param=shared[:256], grad=f(256), m=f(256), v=f(256)), one(param=shared[256:556])])
    g = f(300)
    B.make_adamw_tensors([one(grad=g), one(grad=g)])               # a gradient may be read twice


def test_states_are_read_into_different_memory():
    t = B.make_adamw_tensors(_entries([300, 300], True, False, False))
    a, b, c = (torch.zeros(300, device="cuda") for _ in range(3))
    for m, v in (([a, a], [b, c]), ([a, b], [c, c]), ([a, b], [c, a])):
        with pytest.raises(B.MoeError) as e:
            B.moe_adamw_states_read(t, m, v)
        assert e.value.status == B.MOE_ERR_ARG
    B.moe_adamw_states_write(t, [a, a], [b, b], _status())          # what is only read may be given twice


# ------------------------------------------------------------------------------------------------ together
def test_a_training_step_of_one_block():
    """norm -> gate -> selection -> experts -> Eq. 2 -> norm, its backward pass, and the optimizer: gradients against those of the
    same block in fp64 with the selection held fixed."""
    T, H, N, I, K, budget = 192, 256, 16, 128, 4, 500
    s, ns, i32, bf = B.make_shape(T, H, N, I, 0, K, 1), B.make_norm_shape(T, H, 1), torch.int32, torch.bfloat16
    r, gate = _randn(T, H), _randn(T, 1, seed=1)
    w_in, w_post, w_pre = (1 + 0.1 * _randn(H, seed=k, dtype=torch.float32) for k in (2, 3, 4))
    scale = torch.full((1,), 0.8, device="cuda")
    Wg, W13, W2 = _randn(H, N, seed=5, std=0.1), _randn(N, 2 * I, H, seed=6, std=0.05), _randn(N, H, I, seed=7, std=0.05)
    dn, dr = _randn(T, H, seed=8), _randn(T, H, seed=9)
    st = _status()

    def empty(*shape, dtype=bf):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    # ---- forward
    x = empty(T, H)
    B.moe_block_norm(B.make_norm_shape(T, H), r, None, None, None, None, w_in, None, x)
    scores, idx, top = empty(T, N, dtype=torch.float32), empty(T, K, dtype=i32), empty(T, K, dtype=torch.float32)
    B.moe_gate(s, x, Wg, None, scores, idx, top)
    n_sel, off, tok = empty(T, dtype=i32), empty(N + 1, dtype=i32), empty(budget, dtype=i32)
    wgt, pos = empty(budget, dtype=torch.float32), empty(T, K, dtype=i32)
    B.moe_route(s, idx, top, budget, n_sel, off, tok, wgt, pos, st)
    y_perm, y, r_out, n_out = empty(budget, H), empty(T, H), empty(T, H), empty(T, H)
    ws = B.new_workspace(s, budget)
    B.moe_grouped_ffn(s, x, tok, off, budget, W13, W2, y_perm, st, ws)
    B.moe_combine(s, y_perm, pos, top, n_sel, None, y)
    B.moe_block_norm(ns, r, y, w_post, gate, scale, w_pre, r_out, n_out)
    # ---- backward
    d_r, d_y, d_gate = empty(T, H), empty(T, H), empty(T, 1)
    dw_post, dw_pre, d_scale = empty(H, dtype=torch.float32), empty(H, dtype=torch.float32), empty(1, dtype=torch.float32)
    B.moe_block_norm_backward(ns, r_out, y, w_post, gate, scale, w_pre, dn, dr, d_r, d_y, d_gate, dw_post, dw_pre, d_scale, B.new_norm_workspace(ns))
    d_top, d_yp = empty(T, K, dtype=torch.float32), empty(budget, H)
    B.moe_combine_backward(s, d_y, y_perm, pos, top, n_sel, budget, d_top, d_yp)
    dx_perm, dW13, dW2 = empty(budget, H), torch.empty_like(W13), torch.empty_like(W2)
    B.moe_grouped_ffn_backward(s, x, tok, off, budget, W13, W2, d_yp, dx_perm, dW13, dW2, st, B.new_ffn_backward_workspace(s, budget))
    dx_gate, dWg = empty(T, H), empty(H, N, dtype=torch.float32)
    B.moe_gate_backward(s, x, Wg, scores, idx, n_sel, d_top, None, None, None, dx_gate, dWg, None, st, B.new_router_workspace(s))
    d_x = empty(T, H)
    B.moe_combine(s, dx_perm, pos, torch.ones_like(top), n_sel, dx_gate, d_x)
    d_in, dw_in = empty(T, H), empty(H, dtype=torch.float32)
    B.moe_block_norm_backward(B.make_norm_shape(T, H), r, None, None, None, None, w_in, d_x, d_r, d_in, None, None, None, dw_in, None,
                              B.new_norm_workspace(B.make_norm_shape(T, H)))
    assert int(st) == 0

    # ---- the same in fp64, the selection held fixed
    leaf = {k: v.double().requires_grad_() for k, v in dict(r=r, gate=gate, w_in=w_in, w_post=w_post, w_pre=w_pre, scale=scale, Wg=Wg, W13=W13, W2=W2).items()}
    norm = lambda t, w: w * t / (t.square().mean(1, keepdim=True) + EPS).sqrt()
    xd = norm(leaf["r"], leaf["w_in"])
    p = torch.softmax(xd @ leaf["Wg"], dim=1)
    yd = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    for t_, j in torch.nonzero(torch.arange(K, device="cuda")[None] < n_sel[:, None]).tolist():
        e = int(idx[t_, j])
        u = leaf["W13"][e] @ xd[t_]
        yd = yd.index_add(0, torch.tensor([t_], device="cuda"), (p[t_, e] * (leaf["W2"][e] @ (torch.nn.functional.silu(u[:I]) * u[I:])))[None])
    rd = leaf["r"] + leaf["scale"] * torch.sigmoid(leaf["gate"]) * norm(yd, leaf["w_post"])
    ((rd * dr.double()).sum() + (norm(rd, leaf["w_pre"]) * dn.double()).sum()).backward()
    # bf16 roundings on the way: x, h, y_perm, y, r_out, d_y, d_y_perm, du, dx_perm, d_x, results: about a dozen, independent, at most
    # 2^-8 / sqrt(3) each; twice that for factors that meet in products
    limit = 2 * HALF * np.sqrt(12 / 3)
    for name, got in dict(r=d_in, gate=d_gate, w_in=dw_in, w_post=dw_post, w_pre=dw_pre, scale=d_scale, Wg=dWg, W13=dW13, W2=dW2).items():
        ref = leaf[name].grad
        rel = float((got.double() - ref).norm() / ref.norm())
        assert rel <= limit, (name, rel)

    # ---- update: every weight moves against its gradient's sign (the first step of AdamW without decay is lr sign(g))
    master = [t.float() for t in (Wg, W13, W2, w_in)]
    old = [t.clone() for t in master]
    grads = [dWg, dW13, dW2, dw_in]
    items = [dict(param=m, grad=g, m=torch.zeros_like(m), v=torch.zeros_like(m), copy=c) for m, g, c in zip(master, grads, (Wg, W13, W2, None))]
    B.moe_adamw_step(B.make_adamw_tensors(items), BETA1, BETA2, 1e-20, torch.tensor([1e-3, 1 - BETA1, 1 - BETA2, 1.0], device="cuda"), st)
    for m, o, g in zip(master, old, grads):
        moved, big = m - o, g.abs() > 1e-12
        assert ((moved + 1e-3 * torch.sign(g.float()))[big].abs() <= 1e-6 + 2.0 ** -23 * o.abs()[big]).all()
    assert int(st) == 0 and torch.equal(Wg, master[0].to(bf))
