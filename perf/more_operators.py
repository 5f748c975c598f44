"""The operators for training a budgeted layer, as they are measured: what goes in, their plain form, the calls a user
makes, and their values in 64 bits.

  product   matrix products grouped by expert with ragged sizes: forward, and the gradients of both operands
  experts   the backward pass of the routed experts, from the gradients of their rows to those of the tokens' rows and
            of both weights
  norm      the norm behind a block, its gate and residual scale, the residual and the next block's norm in one step;
            forward and backward
  adamw     an AdamW step over many tensors at once, its states in 32 or in 8 bits
"""
import math
import random

import torch

own = False

BETA1, BETA2, EPS_ADAM = 0.9, 0.999, 1e-8
EPS_NORM = 1e-6
LR, DECAY, STEP, CLIP = 3e-4, 0.1, 7, 0.5     # learning rate, weight decay, steps taken before, factor of a clipped gradient
BLOCK = 256                                   # elements of a state in 8 bits that share a scale
TOP_M, TOP_V = 448.0, 1.9375                  # largest values of the two 8-bit formats


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token's six kept experts, a projection of the 64-expert layer: a product of one row for each, weights read once
        dict(name="product-token", op="product", way="y", E=64, P=6, K=2048, M=2816, tail=0),
        # the same projection on a prefill batch at half its budget, ragged by a skewed router
        dict(name="product-prefill", op="product", way="y", E=64, P=12288, K=2048, M=2816, tail=0),
        # gradient of the rows with 60 experts, an odd number of rows, padding behind the last segment
        dict(name="product-rows-60", op="product", way="dx", E=60, P=4099, K=2048, M=1408, tail=101),
        # gradient of the experts' second weight in 32 bits, as a trainer accumulates it
        dict(name="product-weights", op="product", way="dw32", E=64, P=12288, K=1408, M=2048, tail=0),
        # the experts' backward pass for few tokens: every weight read and every gradient written for three rows an expert
        dict(name="experts-few", op="experts", T=64, H=2048, I=1408, N=64, K=6, kept=3.0),
        # the same for a full training batch of one GPU
        dict(name="experts-batch", op="experts", T=4096, H=2048, I=1408, N=64, K=6, kept=3.0),
        # a served token between two blocks: latency alone
        dict(name="norm-token", op="norm", way="forward", T=1, H=2048, gate=1),
        # the large layer's prefill with a gate for each channel
        dict(name="norm-prefill", op="norm", way="forward", T=8192, H=4096, gate=4096),
        # gradients for an odd batch with one gate a token
        dict(name="norm-back", op="norm", way="backward", T=4099, H=2048, gate=1),
        # the routers of a stack of 26 layers, weights and biases: many small tensors
        dict(name="adamw-routers", op="adamw", sizes="131072*26+64*26", states=32, param="master", grad="f32"),
        # one layer's second expert weights with 32-bit states
        dict(name="adamw-experts", op="adamw", sizes="184549376+5767168", states=32, param="master", grad="bf16"),
        # the same weights with 8-bit states, the states read back as a checkpoint does
        dict(name="adamw-experts-8", op="adamw", sizes="184549376+5767168", states=8, param="master", grad="bf16"),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["product", "experts", "norm", "adamw"])
        c = dict(op=op)
        if op == "product":
            P = _log_int(rng, 1, 16384)
            c.update(way=rng.choice(["y", "dx", "dw16", "dw32"]), E=_log_int(rng, 1, 128), P=P, K=_log_int(rng, 64, 4096, 8),
                     M=_log_int(rng, 64, 4096, 8), tail=rng.choice([0, P // 9]))
        if op == "experts":
            K = rng.randint(1, 8)
            c.update(T=_log_int(rng, 1, 4096), H=_log_int(rng, 256, 4096, 64), I=_log_int(rng, 64, 2816, 64),
                     N=_log_int(rng, 8, 128, 4), K=K, kept=round(rng.uniform(0.5, 1.0) * K, 2))
        if op == "norm":
            H = _log_int(rng, 64, 8192, 8)
            c.update(way=rng.choice(["forward", "backward"]), T=_log_int(rng, 1, 16384), H=H, gate=rng.choice([0, 1, H]))
        if op == "adamw":
            sizes = [_log_int(rng, 1, 1 << 24) for _ in range(_log_int(rng, 1, 64))]
            c.update(sizes="+".join("%d*1" % n for n in sizes), states=rng.choice([8, 32]), param=rng.choice(["master", "bf16"]),
                     grad=rng.choice(["bf16", "f32"]))
        if _cost(c) <= most and all(c != {k: v for k, v in d.items() if k != "name"} for d in listed()):
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 200)


def _sizes(c):
    out = []
    for part in c["sizes"].split("+"):
        n, times = (part.split("*") + ["1"])[:2]
        out += [int(n)] * int(times)
    return out


def _kept(c):
    return max(1, int(c["kept"] * c["T"]))


def _touched(groups, rows):
    """Groups that at least one row falls to, on average."""
    return groups * (1.0 - (1.0 - 1.0 / groups) ** rows)


def work(case):
    """Every input once, every output once; two operations for a multiplication and an addition."""
    c = case
    if c["op"] == "product":
        E, P, K, M = c["E"], c["P"] - c["tail"], c["K"], c["M"]
        if c["way"] in ("dw16", "dw32"):
            moved = 2 * P * (K + M) + (2 if c["way"] == "dw16" else 4) * E * K * M
        else:
            moved = 2 * P * (K + M) + 2 * _touched(E, P) * K * M
        return {"bytes": moved + 4 * (E + 1), "flops": 2 * P * K * M}
    if c["op"] == "experts":
        T, H, I, N, B = c["T"], c["H"], c["I"], c["N"], _kept(c)
        moved = 2 * H * (min(T, B) + 2 * B) + 2 * 3 * I * H * (_touched(N, B) + N) + 4 * (B + N + 1)
        return {"bytes": moved, "flops": 16 * B * H * I}
    if c["op"] == "norm":
        T, H, G = c["T"], c["H"], c["gate"]
        if c["way"] == "forward":
            return {"bytes": 2 * T * (4 * H + G) + 8 * H + 4, "flops": 12 * T * H}
        return {"bytes": 2 * T * (6 * H + 2 * G) + 16 * H + 8, "flops": 40 * T * H}
    n = sum(_sizes(c))
    state = 16 if c["states"] == 32 else 4 + 8 + 16 / BLOCK   # 8 bits: codes both ways, and their values
    param = 8 + 2 if c["param"] == "master" else 4
    return {"bytes": n * (param + (2 if c["grad"] == "bf16" else 4) + state), "flops": 20 * n}


# ------------------------------------------------------------------------------------------------ inputs
def _segments(host, rows, groups):
    """Offsets of ragged segments as a skewed router leaves them: popular groups, rare ones, empty ones."""
    weight = [math.exp(host.gauss(0.0, 0.7)) for _ in range(groups)]
    counts = [0] * groups
    for e in host.choices(range(groups), weights=weight, k=rows):
        counts[e] += 1
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _laid_out(sizes):
    """Where each tensor starts in a buffer that holds all of them; starts are multiples of a block."""
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    return at


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, device="cuda", generator=g) * std).to(dtype)

    op = c["op"]
    s = {"case": c}
    if op == "product":
        E, P, K, M = c["E"], c["P"], c["K"], c["M"]
        s["at"] = _segments(host, P - c["tail"], E)
        s["offsets"] = torch.tensor(s["at"], dtype=torch.int32, device="cuda")
        if c["way"] != "dx":
            s["x"] = normal(P, K)
        if c["way"] != "y":
            s["dy"] = normal(P, M)
        if c["way"] in ("y", "dx"):
            s["W"] = normal(E, M, K, std=0.02)
            s["out"] = torch.zeros(P, M if c["way"] == "y" else K, dtype=torch.bfloat16, device="cuda")
    if op == "experts":
        T, H, I, N, K = c["T"], c["H"], c["I"], c["N"], c["K"]
        B = s["budget"] = _kept(c)
        s["x"], s["W13"], s["W2"] = normal(T, H), normal(N, 2 * I, H, std=0.02), normal(N, H, I, std=0.02)
        s["dy"] = normal(B, H, std=0.1)
        # the budget's pairs: each token's best experts by a profile of favoured ones, the globally best kept
        logits = normal(T, N, dtype=torch.float32) + 0.5 * normal(N, dtype=torch.float32)
        top = torch.topk(torch.softmax(logits, dim=1), K, dim=1)
        keep = torch.topk(top.values.flatten(), B).indices
        pair = torch.sort(top.indices.flatten()[keep] * T + keep // K).values
        s["perm_token"] = (pair % T).to(torch.int32)
        counts = torch.bincount(pair // T, minlength=N)
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["at"] = s["offsets"].tolist()
    if op == "norm":
        T, H, G = c["T"], c["H"], c["gate"]
        s["r"], s["y"] = normal(T, H), normal(T, H, std=0.3)
        s["gate"] = normal(T, G) if G else None
        s["w_post"] = 1.0 + normal(H, std=0.2, dtype=torch.float32)
        s["w_pre"] = 1.0 + normal(H, std=0.2, dtype=torch.float32)
        s["scale"] = torch.full((1,), 0.7, device="cuda")
        if c["way"] == "backward":
            s["dn"], s["dr"] = normal(T, H), normal(T, H)
    if op == "adamw":
        sizes = _sizes(c)
        at = s["at"] = _laid_out(sizes)
        s["sizes"], n = sizes, at[-1]
        # what lies between two tensors is zero on every side
        inside = torch.zeros(n, dtype=torch.bool, device="cuda")
        for k, a in zip(sizes, at):
            inside[a:a + k] = True

        def flat(std, dtype):
            return torch.where(inside, torch.randn(n, device="cuda", generator=g) * std, 0.0).to(dtype)

        s["p"] = flat(0.02, torch.float32 if c["param"] == "master" else torch.bfloat16)
        # gradients of very unlike sizes, as those of rows seldom used are
        size = torch.exp(torch.randn(n // BLOCK, 1, device="cuda", generator=g)).expand(-1, BLOCK).reshape(-1)
        s["g"] = (flat(1e-3, torch.float32) * size).to(torch.bfloat16 if c["grad"] == "bf16" else torch.float32)
        m, v = flat(1e-3, torch.float32) * size, (flat(2e-3, torch.float32) * size).square()
        s["hyper"] = torch.tensor([LR, 1 - BETA1 ** STEP, 1 - BETA2 ** STEP, CLIP], device="cuda")
        if c["states"] == 32:
            s["m"], s["v"] = m, v
        else:
            s["m"], s["m_scale"] = _to_m8(m)
            s["v"], s["v_scale"] = _to_v8(v)
            s["m32"], s["v32"] = torch.zeros_like(m), torch.zeros_like(v)
        if c["param"] == "master":
            s["copy"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        if "lib" not in state:
            _own_buffers(state)
        return {"product": _own_product, "experts": _own_experts, "norm": _own_norm, "adamw": _own_adamw}[op](state)
    return {"product": _plain_product, "experts": _plain_experts, "norm": _plain_norm, "adamw": _plain_adamw}[op](state)


# ---- the framework's calls
def _own_buffers(s):
    """What a program keeps between calls: output buffers, a workspace, the optimizer's list of tensors, the status word."""
    from paper_2604_08133_b200 import binding as B
    c = s["case"]
    op = c["op"]

    def empty(*shape, dtype):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    f32, b16 = torch.float32, torch.bfloat16
    s["lib"] = B
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if op == "product":
        s["shape"] = B.make_grouped_shape(c["P"], c["K"], c["M"], c["E"])
        if c["way"] in ("dw16", "dw32"):
            s["out"] = empty(c["E"], c["M"], c["K"], dtype=b16 if c["way"] == "dw16" else f32)
    if op == "experts":
        s["shape"] = B.make_shape(c["T"], c["H"], c["N"], c["I"], 0, c["K"], 0)
        s["ws"] = B.new_ffn_backward_workspace(s["shape"], s["budget"])
        s["dx"] = torch.empty_like(s["dy"])
        s["dW13"], s["dW2"] = torch.empty_like(s["W13"]), torch.empty_like(s["W2"])
    if op == "norm":
        T, H, G = c["T"], c["H"], c["gate"]
        s["shape"] = B.make_norm_shape(T, H, G, EPS_NORM)
        if c["way"] == "forward":
            s["r_out"], s["n_out"] = torch.empty_like(s["r"]), torch.empty_like(s["r"])
        else:
            s["ws"] = B.new_norm_workspace(s["shape"])
            s["d_r"], s["d_y"] = torch.empty_like(s["r"]), torch.empty_like(s["r"])
            s["d_gate"] = empty(T, G, dtype=b16) if G else None
            s["dw_post"], s["dw_pre"], s["d_scale"] = empty(H, dtype=f32), empty(H, dtype=f32), empty(1, dtype=f32)
    if op == "adamw":
        eight = c["states"] == 8

        def part(name, k):
            a, n = s["at"][k], s["sizes"][k]
            if name not in s:
                return None
            if name.endswith("_scale"):
                return s[name][a // BLOCK:a // BLOCK + -(-n // BLOCK)]
            return s[name][a:a + n]

        count = len(s["sizes"])
        s["tensors"] = B.make_adamw_tensors([
            dict(param=part("p", k), grad=part("g", k), m=part("m", k), v=part("v", k), m_scale=part("m_scale", k),
                 v_scale=part("v_scale", k), copy=part("copy", k), weight_decay=DECAY) for k in range(count)])
        if eight:
            s["m_values"] = [part("m32", k) for k in range(count)]
            s["v_values"] = [part("v32", k) for k in range(count)]


def _own_product(s):
    B, way = s["lib"], s["case"]["way"]
    if way == "y":
        B.moe_grouped_gemm(s["shape"], s["x"], s["offsets"], s["W"], s["out"], s["status"])
    elif way == "dx":
        B.moe_grouped_gemm_dx(s["shape"], s["dy"], s["offsets"], s["W"], s["out"], s["status"])
    else:
        B.moe_grouped_gemm_dw(s["shape"], s["dy"], s["x"], s["offsets"], s["out"], s["status"])
    return s["out"]


def _own_experts(s):
    s["lib"].moe_grouped_ffn_backward(s["shape"], s["x"], s["perm_token"], s["offsets"], s["budget"], s["W13"], s["W2"], s["dy"],
                                      s["dx"], s["dW13"], s["dW2"], s["status"], s["ws"])
    return s["dx"], s["dW13"], s["dW2"]


def _own_norm(s):
    B = s["lib"]
    if s["case"]["way"] == "forward":
        B.moe_block_norm(s["shape"], s["r"], s["y"], s["w_post"], s["gate"], s["scale"], s["w_pre"], s["r_out"], s["n_out"])
        return s["r_out"], s["n_out"]
    B.moe_block_norm_backward(s["shape"], s["r"], s["y"], s["w_post"], s["gate"], s["scale"], s["w_pre"], s["dn"], s["dr"],
                              s["d_r"], s["d_y"], s["d_gate"], s["dw_post"], s["dw_pre"], s["d_scale"], s["ws"])
    return s["d_r"], s["d_y"], s["d_gate"], s["dw_post"], s["dw_pre"], s["d_scale"]


def _own_adamw(s):
    B = s["lib"]
    B.moe_adamw_step(s["tensors"], BETA1, BETA2, EPS_ADAM, s["hyper"], s["status"])
    if s["case"]["states"] == 32:
        return s["p"], s["m"], s["v"], s.get("copy")
    B.moe_adamw_states_read(s["tensors"], s["m_values"], s["v_values"])
    return s["p"], s["m32"], s["v32"], s.get("copy")


# ---- the plain forms
def _padded_index(s):
    """Row numbers by group, [E, longest], and which of them are rows of the group; the others name the row behind the last."""
    at, P = s["at"], s["case"].get("P", s.get("budget"))
    longest = max(max(b - a for a, b in zip(at, at[1:])), 1)
    first, count = s["offsets"][:-1, None].long(), (s["offsets"][1:] - s["offsets"][:-1])[:, None]
    j = torch.arange(longest, device="cuda")[None, :]
    inside = j < count
    return torch.where(inside, first + j, P)


def _by_group(rows, index):
    """[E, longest, columns] in 32 bits, zeros where a group has no row."""
    more = torch.cat([rows.float(), rows.new_zeros(1, rows.shape[1], dtype=torch.float32)])
    return more[index]


def _to_rows(groups, index, rows):
    out = groups.new_zeros(rows + 1, groups.shape[2])
    return out.index_copy(0, index.flatten(), groups.flatten(0, 1))[:rows]


def _plain_product(s):
    c = s["case"]
    index = _padded_index(s)
    if c["way"] == "y":
        y = torch.bmm(_by_group(s["x"], index), s["W"].float().transpose(1, 2))
        return _to_rows(y, index, c["P"]).to(torch.bfloat16)
    if c["way"] == "dx":
        dx = torch.bmm(_by_group(s["dy"], index), s["W"].float())
        return _to_rows(dx, index, c["P"]).to(torch.bfloat16)
    dW = torch.bmm(_by_group(s["dy"], index).transpose(1, 2), _by_group(s["x"], index))
    return dW.to(torch.bfloat16) if c["way"] == "dw16" else dW


def _plain_experts(s):
    index = _padded_index(s)
    x, dy = _by_group(s["x"][s["perm_token"].long()], index), _by_group(s["dy"], index)
    W13, W2 = s["W13"].float(), s["W2"].float()
    gate, up = torch.bmm(x, W13.transpose(1, 2)).chunk(2, dim=2)
    sg = 1.0 / (1.0 + torch.exp(-gate))
    silu = gate * sg
    dh = torch.bmm(dy, W2)
    dW2 = torch.bmm(dy.transpose(1, 2), silu * up)
    du = torch.cat([dh * up * sg * (1.0 + gate * (1.0 - sg)), dh * silu], dim=2)
    dx = _to_rows(torch.bmm(du, W13), index, s["budget"])
    dW13 = torch.bmm(du.transpose(1, 2), x)
    return dx.to(torch.bfloat16), dW13.to(torch.bfloat16), dW2.to(torch.bfloat16)


def _plain_norm(s):
    c = s["case"]
    y = s["y"].float()
    sg = 1.0 / (1.0 + torch.exp(-s["gate"].float())) if c["gate"] else torch.ones(1, 1, device="cuda")
    inv_y = 1.0 / torch.sqrt((y * y).mean(1, keepdim=True) + EPS_NORM)
    y_hat = y * inv_y
    if c["way"] == "forward":
        r = (s["r"].float() + s["scale"] * sg * (y_hat * s["w_post"])).to(torch.bfloat16)
        back = r.float()
        inv_r = 1.0 / torch.sqrt((back * back).mean(1, keepdim=True) + EPS_NORM)
        return r, (back * inv_r * s["w_pre"]).to(torch.bfloat16)
    r, dn = s["r"].float(), s["dn"].float()
    inv_r = 1.0 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS_NORM)
    r_hat = r * inv_r
    d_hat = dn * s["w_pre"]
    d_r = s["dr"].float() + inv_r * (d_hat - r_hat * (d_hat * r_hat).mean(1, keepdim=True))
    p = y_hat * s["w_post"]
    d_p = d_r * s["scale"] * sg
    d_yhat = d_p * s["w_post"]
    d_y = inv_y * (d_yhat - y_hat * (d_yhat * y_hat).mean(1, keepdim=True))
    # long sums in 64 bits
    d_scale = (d_r * sg * p).sum(dtype=torch.float64).float().reshape(1)
    dw_post, dw_pre = (d_p * y_hat).sum(0, dtype=torch.float64).float(), (dn * r_hat).sum(0, dtype=torch.float64).float()
    d_gate = None
    if c["gate"]:
        d_gate = d_r * s["scale"] * p * (sg * (1.0 - sg))
        d_gate = (d_gate if c["gate"] > 1 else d_gate.sum(1, keepdim=True)).to(torch.bfloat16)
    return d_r.to(torch.bfloat16), d_y.to(torch.bfloat16), d_gate, dw_post, dw_pre, d_scale


def _scale_of(largest, top):
    """The block's scale and the factor to its codes; a block below 2^-100 counts as zero."""
    used = largest >= 2.0 ** -100
    tops = torch.full_like(largest, top)
    safe = torch.where(used, largest, 1.0)
    return torch.where(used, safe / tops, 0.0), torch.where(used, tops / safe, 0.0)


def _to_m8(m):
    blocks = m.view(-1, BLOCK)
    scale, factor = _scale_of(blocks.abs().amax(1, keepdim=True), TOP_M)
    return (blocks * factor).to(torch.float8_e4m3fn).view(torch.uint8).view(-1), scale.view(-1)


def _from_m8(codes, scale):
    return (codes.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _to_v8(v):
    """sqrt(v) with four bits of exponent and four of mantissa, to the nearest even; above zero it stays above zero."""
    u = torch.sqrt(v).view(-1, BLOCK)
    scale, factor = _scale_of(u.amax(1, keepdim=True), TOP_V)
    bits = (u * factor).view(torch.int32)
    code = ((bits + 0x3FFFF + ((bits >> 19) & 1)) >> 19) - (112 << 4)
    code = torch.where((u > 0) & (scale > 0), code.clamp(1, 255), 0)
    return code.to(torch.uint8).view(-1), scale.view(-1)


def _from_v8(codes, scale):
    code = codes.to(torch.int32).view(-1, BLOCK)
    u = torch.where(code > 0, ((code + (112 << 4)) << 19).view(torch.float32), 0.0) * scale[:, None]
    return (u * u).view(-1)


def _plain_adamw(s):
    eight = s["case"]["states"] == 8
    lr, bias1, bias2, clip = s["hyper"].unbind()
    m, v = (_from_m8(s["m"], s["m_scale"]), _from_v8(s["v"], s["v_scale"])) if eight else (s["m"], s["v"])
    # every product and sum of the states rounded by itself: the 8-bit codes are defined by these steps
    g = s["g"].float() * clip
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * (1 - BETA2)) * g
    p = s["p"].float()
    p = p * (1.0 - lr * DECAY) - (lr / bias1) * (m / (torch.sqrt(v) / torch.sqrt(bias2) + EPS_ADAM))
    s["p"].copy_(p)
    if "copy" in s:
        s["copy"].copy_(p)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return s["p"], s["m"], s["v"], s.get("copy")
    (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _to_m8(m), _to_v8(v)
    return s["p"], _from_m8(s["m"], s["m_scale"]), _from_v8(s["v"], s["v_scale"]), s.get("copy")


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    op, f64 = c["op"], torch.float64
    if op == "product":
        E, at = c["E"], s["at"]
        if c["way"] in ("dw16", "dw32"):
            out = torch.zeros(E, c["M"], c["K"], dtype=f64, device="cuda")
            for e in range(E):
                out[e] = torch.einsum("pm,pk->mk", s["dy"][at[e]:at[e + 1]].double(), s["x"][at[e]:at[e + 1]].double())
            return out
        out = torch.zeros(c["P"], c["M"] if c["way"] == "y" else c["K"], dtype=f64, device="cuda")
        for e in range(E):
            W = s["W"][e].double()
            rows = slice(at[e], at[e + 1])
            out[rows] = s["x"][rows].double() @ W.T if c["way"] == "y" else s["dy"][rows].double() @ W
        return out
    if op == "experts":
        at, I = s["at"], c["I"]
        dx = torch.zeros(s["budget"], c["H"], dtype=f64, device="cuda")
        dW13 = torch.zeros(s["W13"].shape, dtype=f64, device="cuda")
        dW2 = torch.zeros(s["W2"].shape, dtype=f64, device="cuda")
        for e in range(c["N"]):
            x = s["x"][s["perm_token"][at[e]:at[e + 1]].long()].double()
            dy, W13, W2 = s["dy"][at[e]:at[e + 1]].double(), s["W13"][e].double(), s["W2"][e].double()
            u = x @ W13.T
            u1, u3 = u[:, :I], u[:, I:]
            silu = torch.nn.functional.silu(u1)
            # d silu / d u = sigmoid(u) + silu(u) (1 - sigmoid(u)), and 1 - sigmoid(u) = sigmoid(-u)
            slope = torch.sigmoid(u1) + silu * torch.sigmoid(-u1)
            dh = dy @ W2
            du = torch.cat([dh * u3 * slope, dh * silu], dim=1)
            dx[at[e]:at[e + 1]] = du @ W13
            dW13[e], dW2[e] = du.T @ x, dy.T @ (silu * u3)
        return dx, dW13, dW2
    if op == "norm":
        d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
        sg = torch.sigmoid(d["gate"]) if c["gate"] else torch.ones(c["T"], 1, dtype=f64, device="cuda")
        H = c["H"]
        inv_y = ((d["y"] ** 2).sum(1) / H + EPS_NORM) ** -0.5
        if c["way"] == "forward":
            r = d["r"] + d["scale"] * sg * d["w_post"] * d["y"] * inv_y[:, None]
            # the next norm sees the residual as it is stored
            back = r.to(torch.bfloat16).double()
            return r, d["w_pre"] * back * ((back ** 2).sum(1) / H + EPS_NORM)[:, None] ** -0.5
        inv_r = ((d["r"] ** 2).sum(1) / H + EPS_NORM) ** -0.5
        a = d["dn"] * d["w_pre"]
        d_r = d["dr"] + inv_r[:, None] * a - d["r"] * (inv_r ** 3 * (a * d["r"]).sum(1) / H)[:, None]
        b = d["scale"] * sg * d_r * d["w_post"]
        d_y = inv_y[:, None] * b - d["y"] * (inv_y ** 3 * (b * d["y"]).sum(1) / H)[:, None]
        y_hat, r_hat = d["y"] * inv_y[:, None], d["r"] * inv_r[:, None]
        d_gate = None
        if c["gate"]:
            d_gate = d_r * d["scale"] * y_hat * d["w_post"]
            d_gate = (d_gate if c["gate"] > 1 else d_gate.sum(1, keepdim=True)) * sg * (1 - sg)
        return (d_r, d_y, d_gate, (d_r * d["scale"] * sg * y_hat).sum(0), (d["dn"] * r_hat).sum(0),
                (d_r * sg * y_hat * d["w_post"]).sum().reshape(1))
    g = s["g"].double() * CLIP
    if c["states"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m = s["m"].view(torch.float8_e4m3fn).double() * s["m_scale"].double().repeat_interleave(BLOCK)
        code = s["v"].double()
        u = (1 + code.remainder(16) / 16) * 2.0 ** ((code / 16).floor() - 15) * s["v_scale"].double().repeat_interleave(BLOCK)
        v = torch.where(code > 0, u * u, 0.0)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    bias1, bias2 = 1 - BETA1 ** STEP, 1 - BETA2 ** STEP
    p = s["p"].double() * (1 - LR * DECAY) - LR * (m / bias1) / ((v / bias2).sqrt() + EPS_ADAM)
    copy = p if "copy" in s else None
    # the codes of 8-bit states follow from the operator's own 32-bit steps: 64 bits would cross borders between two codes
    return (p, m, v, copy) if c["states"] == 32 else (p, None, None, copy)
