"""The operators for adapting a frozen budgeted layer, as they are measured: what goes in, their plain form, the
calls a user makes, and their values in 64 bits.

  balance   counts of the kept pairs per expert and sequence, the balance loss over them and its gradient with respect
            to the gate's logits
  gate      the gate's backward pass: from the gradients of the kept scores (and the balance loss) to the logits, the
            tokens, W_gate and the gate bias
  combine   the gradients of Eq. 2's weighted sum with respect to the scores and the experts' rows
  adapter   a projection with a low-rank adapter per request beside the shared weight
  shared    the shared experts with such adapters beside both of their projections
"""
import math
import random

import torch

own = False

ALPHA = 0.01   # weight of the balance loss


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of the 64-expert layer at half its budget: a router update from few tokens, latency bound
        dict(name="balance-decode", op="balance", T=64, N=64, K=6, kept=3.0, n_seq=1, tail=0),
        # a packed training batch: ragged sequences, padding behind the last one
        dict(name="balance-packed", op="balance", T=65521, N=64, K=6, kept=3.0, n_seq=37, tail=803),
        # the gate's gradient for one small batch
        dict(name="gate-small", op="gate", T=64, H=2048, N=64, K=6, kept=3.0, n_seq=1, tail=0),
        # 60 experts (no multiple of eight), an odd packed batch, padded at its end
        dict(name="gate-packed-60", op="gate", T=4099, H=2048, N=60, K=4, kept=2.5, n_seq=9, tail=101),
        # the large layer with few experts: the bytes of x and of its gradient decide
        dict(name="gate-wide-8", op="gate", T=8192, H=4096, N=8, K=2, kept=1.5, n_seq=4, tail=0),
        # Eq. 2's gradient for a decode batch and for a prefill batch
        dict(name="combine-decode", op="combine", T=64, H=2048, N=64, K=6, kept=3.0),
        dict(name="combine-prefill", op="combine", T=4096, H=2048, N=64, K=6, kept=3.0),
        # one request's single token
        dict(name="adapter-token", op="adapter", T=1, K=2048, M=4096, n=4, r=16, requests=1),
        # a decode batch, every request with its own adapter
        dict(name="adapter-decode", op="adapter", T=64, K=2048, M=2816, n=48, r=16, requests=64),
        # a prefill of eleven requests of ragged length
        dict(name="adapter-prefill", op="adapter", T=4096, K=2048, M=2816, n=8, r=64, requests=11),
        # the layer's two shared experts with adapters: decode and prefill
        dict(name="shared-decode", op="shared", T=64, H=2048, I=1408, S=2, n=32, r=16, requests=64),
        dict(name="shared-prefill", op="shared", T=2045, H=2048, I=1408, S=2, n=8, r=32, requests=7),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["balance", "gate", "combine", "adapter", "shared"])
        T = _log_int(rng, 1, 65536 if op == "balance" else 8192)
        N = _log_int(rng, 8, 128, 4)
        K = rng.randint(1, min(N, 16))
        c = dict(op=op, T=T)
        if op in ("balance", "gate", "combine"):
            c.update(N=N, K=K, kept=round(rng.uniform(0.5, 1.0) * K, 2))
        if op in ("gate", "combine"):
            c["H"] = _log_int(rng, 256, 4096, 64)
        if op in ("balance", "gate"):
            c.update(n_seq=_log_int(rng, 1, max(1, min(64, T // 2))), tail=rng.choice([0, T // 9]))
        if op in ("adapter", "shared"):
            c.update(n=_log_int(rng, 1, 64), r=8 * rng.randint(1, 16))
            c["requests"] = T if T <= 128 else _log_int(rng, 1, 32)
        if op == "adapter":
            c.update(K=_log_int(rng, 256, 8192, 8), M=_log_int(rng, 256, 8192, 8))
        if op == "shared":
            c.update(H=_log_int(rng, 256, 4096, 64), I=_log_int(rng, 256, 2816, 64), S=rng.choice([1, 2]))
        if _cost(c) <= most and all(c != {k: v for k, v in d.items() if k != "name"} for d in listed()):
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _request_adapters(c):
    """The adapter of each request; every eighth request has none."""
    return [-1 if k % 8 == 7 else k % c["n"] for k in range(c["requests"])]


def _kept(c):
    return max(1, int(c["kept"] * c["T"]))


def work(case):
    """Every input once, every output once; two operations for a multiplication and an addition."""
    c = case
    T = c["T"]
    if c["op"] == "balance":
        N, K, n_seq = c["N"], c["K"], c["n_seq"]
        return {"bytes": 4 * (2 * T * N + T * K + T + 2 * n_seq * N + n_seq + 2), "flops": 5 * T * N}
    if c["op"] == "gate":
        H, N, K, n_seq = c["H"], c["N"], c["K"], c["n_seq"]
        moved = 4 * (2 * T * N + 2 * T * K + T + n_seq * N) + 2 * (2 * T * H + H * N) + 4 * (H * N + N)
        return {"bytes": moved, "flops": 4 * T * H * N + 5 * T * N}
    if c["op"] == "combine":
        H, K, B = c["H"], c["K"], _kept(c)
        return {"bytes": 2 * H * (T + 2 * B) + 4 * (3 * T * K + T), "flops": 3 * B * H}
    used = len({a for a in _request_adapters(c) if a >= 0})
    if c["op"] == "adapter":
        K, M, r = c["K"], c["M"], c["r"]
        return {"bytes": 2 * (M * K + T * (K + M) + used * r * (K + M)) + 4 * (T + c["n"]),
                "flops": 2 * T * (K * M + r * (K + M))}
    H, I, S, r = c["H"], c["I"], c["S"], c["r"]
    return {"bytes": 2 * (3 * S * I * H + 2 * T * H + used * r * (2 * H + 3 * S * I)) + 4 * (T + c["n"]),
            "flops": 2 * T * (3 * S * I * H + r * (2 * H + 3 * S * I))}


# ------------------------------------------------------------------------------------------------ inputs
def _cuts(rng, total, parts):
    """`parts` ragged lengths that add up to `total`, as offsets; the third part of four and more is empty."""
    at = [0] + sorted(rng.randint(0, total) for _ in range(parts - 1)) + [total]
    if parts >= 4:
        at[3] = at[2]
    return at


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, device="cuda", generator=g) * std).to(dtype)

    T, op = c["T"], c["op"]
    s = {"case": c}
    if op in ("balance", "gate", "combine"):
        N, K = c["N"], c["K"]
        # logits with a standard deviation of about one and a profile of favoured experts, as a trained gate has
        logits = normal(T, N, dtype=torch.float32) + 0.5 * normal(N, dtype=torch.float32)
        s["scores"] = torch.softmax(logits, dim=1)
        top = torch.topk(s["scores"], K, dim=1)
        s["topk_score"], s["topk_idx"] = top.values.contiguous(), top.indices.to(torch.int32)
        # the kept counts of a budget of `kept` pairs a token: the globally largest scores, all of them rows' prefixes
        budget = _kept(c)
        flat = s["topk_score"].flatten()
        n = torch.zeros(T, dtype=torch.int32, device="cuda")
        keep = torch.topk(flat, budget).indices
        s["n_sel"] = n.index_add_(0, keep // K, torch.ones_like(keep, dtype=torch.int32))
        s["budget"] = budget
    if op in ("balance", "gate"):
        at = _cuts(host, T - c["tail"], c["n_seq"])
        s["seq_offsets"] = torch.tensor(at, dtype=torch.int32, device="cuda")
    if op == "gate":
        H, N, n_seq = c["H"], c["N"], c["n_seq"]
        s["x"] = normal(T, H)
        s["W_gate"] = normal(H, N, std=0.02)
        s["d_topk_score"] = normal(T, K, std=0.1, dtype=torch.float32)
        s["coef"] = normal(n_seq, N, std=0.01, dtype=torch.float32).abs()   # of the balance loss, for these sequences
    if op == "combine":
        H = c["H"]
        s["d_out"] = normal(T, H)
        s["y_perm"] = normal(max(budget, 1), H, std=0.5)
        # list positions expert-ascending, token-ascending inside an expert
        kept = torch.arange(K, device="cuda")[None, :] < s["n_sel"][:, None]
        key = torch.where(kept, s["topk_idx"].long(), N) * T + torch.arange(T, device="cuda")[:, None]
        pos = torch.empty(T * K, dtype=torch.int32, device="cuda")
        pos[torch.argsort(key.flatten())] = torch.arange(T * K, dtype=torch.int32, device="cuda")
        s["pair_pos"] = torch.where(kept, pos.view(T, K), -1).contiguous()
    if op in ("adapter", "shared"):
        n, r = c["n"], c["r"]
        who = _request_adapters(c)
        if c["requests"] == T:
            host.shuffle(who)
            ids = who
        else:
            at = _cuts(host, T, c["requests"])
            ids = [a for k, a in enumerate(who) for _ in range(at[k], at[k + 1])]
        s["adapter_id"] = torch.tensor(ids, dtype=torch.int32, device="cuda")
        s["scale"] = torch.tensor([host.choice([0.5, 1.0, 2.0]) for _ in range(n)], dtype=torch.float32, device="cuda")
    if op == "adapter":
        K, M = c["K"], c["M"]
        s["x"], s["W"] = normal(T, K), normal(M, K, std=0.02)
        s["A"], s["B"] = normal(n, r, K, std=K ** -0.5), normal(n, M, r, std=0.1)
    if op == "shared":
        H, I, S = c["H"], c["I"], c["S"]
        s["x"] = normal(T, H)
        s["Wsh13"], s["Wsh2"] = normal(S, 2 * I, H, std=0.02), normal(S, H, I, std=0.02)
        s["A13"], s["B13"] = normal(n, r, H, std=H ** -0.5), normal(n, S * 2 * I, r, std=0.1)
        s["A2"], s["B2"] = normal(n, r, S * I, std=(S * I) ** -0.5), normal(n, H, r, std=0.1)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        if "status" not in state:
            _own_buffers(state)
        if op == "balance":
            return _own_balance(state)
        if op == "gate":
            return _own_gate(state)
        if op == "combine":
            return _own_combine(state)
        return _own_adapter(state) if op == "adapter" else _own_shared(state)
    if op == "balance":
        return _plain_balance(state)
    if op == "gate":
        return _plain_gate(state)
    if op == "combine":
        return _plain_combine(state)
    return _plain_adapter(state) if op == "adapter" else _plain_shared(state)


# ---- the framework's calls
def _own_buffers(s):
    """What a program keeps between calls: output buffers, a workspace and the status word."""
    from paper_2604_08133_b200 import binding as B
    c = s["case"]
    T, op = c["T"], c["op"]
    f32, i32, b16 = torch.float32, torch.int32, torch.bfloat16

    def empty(*shape, dtype):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s["lib"] = B
    s["status"] = torch.zeros(1, dtype=i32, device="cuda")
    if op in ("balance", "gate", "combine"):
        N, K = c["N"], c["K"]
        H = c.get("H", 64)
        s["shape"] = B.make_shape(T, H, N, 64, 0, K, 0)
    if op in ("balance", "gate"):
        n_seq = c["n_seq"]
        s["ws"] = B.new_router_workspace(s["shape"], n_seq)
        s["d_logits"] = empty(T, N, dtype=f32)
    if op == "balance":
        s["counts"], s["coef"] = empty(n_seq, N, dtype=i32), empty(n_seq, N, dtype=f32)
        s["loss"] = empty(1, dtype=f32)
    if op == "gate":
        s["dx"], s["dW"] = empty(T, H, dtype=b16), empty(H, N, dtype=f32)
        s["d_bias"] = empty(N, dtype=f32)
    if op == "combine":
        s["d_score"], s["d_y"] = empty(T, K, dtype=f32), torch.empty_like(s["y_perm"])
    if op == "adapter":
        s["shape"] = B.make_adapter_shape(T, c["K"], c["M"], c["n"], c["r"])
        s["ws"] = B.new_adapter_workspace(s["shape"])
        s["y"] = empty(T, c["M"], dtype=b16)
    if op == "shared":
        s["shape"] = B.make_shape(T, c["H"], 8, c["I"], c["S"], 1, 0)
        s["ws"] = B.new_shared_adapted_workspace(s["shape"], c["n"], c["r"])
        s["y"] = empty(T, c["H"], dtype=b16)


def _own_balance(s):
    B = s["lib"]
    B.moe_balance_loss(s["shape"], s["scores"], s["topk_idx"], s["n_sel"], s["seq_offsets"], ALPHA, s["counts"], s["coef"],
                       s["loss"], s["status"], s["ws"])
    B.moe_gate_backward(s["shape"], None, None, s["scores"], s["topk_idx"], None, None, s["coef"], s["seq_offsets"],
                        s["d_logits"], None, None, None, s["status"], s["ws"])
    return s["counts"], s["loss"], s["coef"], s["d_logits"]


def _own_gate(s):
    s["lib"].moe_gate_backward(s["shape"], s["x"], s["W_gate"], s["scores"], s["topk_idx"], s["n_sel"], s["d_topk_score"],
                               s["coef"], s["seq_offsets"], s["d_logits"], s["dx"], s["dW"], s["d_bias"], s["status"], s["ws"])
    return s["d_logits"], s["dx"], s["dW"], s["d_bias"]


def _own_combine(s):
    s["lib"].moe_combine_backward(s["shape"], s["d_out"], s["y_perm"], s["pair_pos"], s["topk_score"], s["n_sel"], s["budget"],
                                  s["d_score"], s["d_y"])
    return s["d_score"], s["d_y"]


def _own_adapter(s):
    s["lib"].moe_adapter_linear(s["shape"], s["x"], s["W"], s["A"], s["B"], s["scale"], s["adapter_id"], s["y"], s["status"],
                                s["ws"])
    return s["y"]


def _own_shared(s):
    s["lib"].moe_shared_ffn_adapted(s["shape"], s["x"], s["Wsh13"], s["Wsh2"], s["A13"], s["B13"], s["A2"], s["B2"], s["scale"],
                                    s["adapter_id"], s["y"], s["status"], s["ws"])
    return s["y"]


# ---- the plain forms
def _sequence_of_rows(offsets, T):
    """The sequence of each row (the last whose start is not behind it) and whether the row lies in one at all."""
    t = torch.arange(T, device=offsets.device, dtype=offsets.dtype)
    seq = torch.searchsorted(offsets, t, right=True) - 1
    inside = (t >= offsets[0]) & (t < offsets[-1])
    return seq.clamp(0, offsets.numel() - 2), inside


def _plain_logit_gradient(scores, d_scores, inside):
    d = scores * (d_scores - (scores * d_scores).sum(1, keepdim=True))
    return torch.where(inside[:, None], d, 0.0)


def _plain_balance(s):
    c = s["case"]
    N, K, n_seq = c["N"], c["K"], c["n_seq"]
    scores, offsets = s["scores"], s["seq_offsets"]
    seq, inside = _sequence_of_rows(offsets, c["T"])
    kept = (torch.arange(K, device="cuda")[None, :] < s["n_sel"][:, None]) & inside[:, None]
    slot = seq[:, None] * N + s["topk_idx"]
    counts = torch.zeros(n_seq * N, dtype=torch.int64, device="cuda")
    counts = counts.index_add(0, slot.flatten(), kept.flatten().long()).view(n_seq, N)
    # long sums of scores in 64 bits
    total = torch.zeros(n_seq, N, dtype=torch.float64, device="cuda")
    total = total.index_add(0, seq, torch.where(inside[:, None], scores, 0.0).double())
    rows = (offsets[1:] - offsets[:-1]).float()[:, None]
    pairs = counts.sum(1, keepdim=True).float()
    share = ALPHA * N / n_seq * counts.float() / (pairs * rows).clamp(min=1.0)
    loss = (share * total.float()).sum().reshape(1)
    d_logits = _plain_logit_gradient(scores, share[seq], inside)
    return counts.to(torch.int32), loss, share, d_logits


def _plain_gate(s):
    c = s["case"]
    K = c["K"]
    seq, inside = _sequence_of_rows(s["seq_offsets"], c["T"])
    kept = torch.arange(K, device="cuda")[None, :] < s["n_sel"][:, None]
    d_scores = s["coef"][seq].scatter_add(1, s["topk_idx"].long(), torch.where(kept, s["d_topk_score"], 0.0))
    d_logits = _plain_logit_gradient(s["scores"], d_scores, inside)
    dx = d_logits @ s["W_gate"].float().T
    dW = torch.where(inside[:, None], s["x"], 0).float().T @ d_logits
    return d_logits, dx.to(torch.bfloat16), dW, d_logits.sum(0)


def _plain_combine(s):
    K = s["case"]["K"]
    d_out, y = s["d_out"].float(), s["y_perm"].float()
    kept = torch.arange(K, device="cuda")[None, :] < s["n_sel"][:, None]
    pos = s["pair_pos"].long().clamp(min=0)
    d_score = torch.where(kept, (y[pos] * d_out[:, None, :]).sum(2), 0.0)
    rows = (s["topk_score"][:, :, None] * d_out[:, None, :])[kept]
    d_y = torch.zeros_like(y).index_copy(0, pos[kept], rows)
    return d_score, d_y.to(torch.bfloat16)


def _plain_delta(x, A, B, scale, ids):
    """scale * (x A^T) B^T with each row's own adapter: every adapter's inner values, the others' zeroed, one product."""
    n, r, K = A.shape
    inner = (x @ A.float().reshape(n * r, K).T).view(-1, n, r) * scale[None, :, None]
    mine = ids[:, None] == torch.arange(n, device=ids.device, dtype=ids.dtype)[None, :]
    inner = torch.where(mine[:, :, None], inner, 0.0).view(-1, n * r)
    return inner @ B.float().permute(0, 2, 1).reshape(n * r, B.shape[1])


def _plain_adapter(s):
    x = s["x"].float()
    y = x @ s["W"].float().T + _plain_delta(x, s["A"], s["B"], s["scale"], s["adapter_id"])
    return y.to(torch.bfloat16)


def _plain_shared(s):
    c = s["case"]
    T, H, I, S = c["T"], c["H"], c["I"], c["S"]
    x = s["x"].float()
    u = x @ s["Wsh13"].float().view(S * 2 * I, H).T + _plain_delta(x, s["A13"], s["B13"], s["scale"], s["adapter_id"])
    gate, up = u.view(T, S, 2, I).unbind(2)
    h = (gate / (1.0 + torch.exp(-gate)) * up).reshape(T, S * I)
    W2 = s["Wsh2"].float().permute(1, 0, 2).reshape(H, S * I)
    y = h @ W2.T + _plain_delta(h, s["A2"], s["B2"], s["scale"], s["adapter_id"])
    return y.to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    T, op = c["T"], c["op"]
    f64 = torch.float64
    if op in ("balance", "gate"):
        at = s["seq_offsets"].tolist()
        N, K, n_seq = c["N"], c["K"], c["n_seq"]
        p = s["scores"].double()
        idx, n_sel = s["topk_idx"].long(), s["n_sel"]
        g = torch.zeros(T, N, dtype=f64, device="cuda")
        valid = torch.zeros(T, 1, dtype=f64, device="cuda")
        valid[at[0]:at[-1]] = 1.0
    if op == "balance":
        counts = torch.zeros(n_seq, N, dtype=f64, device="cuda")
        coef = torch.zeros(n_seq, N, dtype=f64, device="cuda")
        loss = torch.zeros((), dtype=f64, device="cuda")
        for b in range(n_seq):
            lo, hi = at[b], at[b + 1]
            for j in range(K if hi > lo else 0):
                counts[b] += torch.bincount(idx[lo:hi, j][n_sel[lo:hi] > j], minlength=N)
            if counts[b].sum() > 0:
                f = N * counts[b] / counts[b].sum()
                loss += ALPHA / n_seq * (f * p[lo:hi].mean(0)).sum()
                coef[b] = ALPHA / n_seq * f / (hi - lo)
                g[lo:hi] = coef[b]
        d = p * (g - (g * p).sum(1, keepdim=True)) * valid
        return None, loss.reshape(1), coef, d
    if op == "gate":
        for b in range(n_seq):
            g[at[b]:at[b + 1]] = s["coef"][b].double()
        for j in range(K):
            keep = (n_sel > j).double()[:, None]
            g += torch.nn.functional.one_hot(idx[:, j], N) * keep * s["d_topk_score"][:, j:j + 1].double()
        d = p * (g - (g * p).sum(1, keepdim=True)) * valid
        return d, d @ s["W_gate"].double().T, (s["x"].double() * valid).T @ d, d.sum(0)
    if op == "combine":
        d_out, y = s["d_out"].double(), s["y_perm"].double()
        d_score = torch.zeros(T, c["K"], dtype=f64, device="cuda")
        d_y = torch.zeros_like(y)
        for j in range(c["K"]):
            t = torch.nonzero(s["n_sel"] > j).flatten()
            q = s["pair_pos"][t, j].long()
            d_score[t, j] = torch.einsum("th,th->t", d_out[t], y[q])
            d_y[q] = s["topk_score"][t, j, None].double() * d_out[t]
        return d_score, d_y

    def adapted(x, W, A, B):
        y = x @ W.double().T
        for a in range(c["n"]):
            t = torch.nonzero(s["adapter_id"] == a).flatten()
            y[t] += float(s["scale"][a]) * ((x[t] @ A[a].double().T) @ B[a].double().T)
        return y

    x = s["x"].double()
    if op == "adapter":
        return adapted(x, s["W"], s["A"], s["B"])
    H, I, S = c["H"], c["I"], c["S"]
    u = adapted(x, s["Wsh13"].reshape(-1, H), s["A13"], s["B13"])
    h = torch.cat([torch.nn.functional.silu(u[:, 2 * k * I:(2 * k + 1) * I]) * u[:, (2 * k + 1) * I:(2 * k + 2) * I]
                   for k in range(S)], dim=1)
    return adapted(h, torch.cat(list(s["Wsh2"]), dim=1), s["A2"], s["B2"])
