"""The operators of a mixture-of-experts layer trained and served in float8, as cases that can be timed and compared.

Four operators that run one behind the other in such a layer, and the step that uses their gradients:

  route     the router's choice: softmax over the experts' logits, the k largest (ties to the lower expert), the
            expert-ordered row lists that the products read; backward: the gradient of the logits.
  grouped   the experts' float8 linear layers over rows grouped by expert, with ragged group sizes: the rowwise recipe's
            forward, its two backward products, and the forward against weights quantized once.
  combine   the gate-weighted sum of each token's expert outputs; backward: gradients of the outputs and of the gates.
  adamw     the AdamW step over many tensors, with moments in 32 bits or in 8 (e4m3 in blocks of 256 with one power-of-two
            scale each; of the second moment the square root).

``own`` false computes them in elementary torch operations in 32 bits, true through the entry points of
``paper_2507_16099_amd``.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
FMAX = {E4M3: 448.0, E5M2: 57344.0}
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
STATE_BLOCK = 256
HYPER = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.1, "step": 1000}


def _route(T, E, k, *, dtype="fp32", renorm=True, mask=True, train=True):
    return {"op": "route", "T": T, "E": E, "k": k, "dtype": dtype, "renorm": renorm, "mask": mask, "train": train}


def _grouped(mode, T, E, k, K, N, *, pow2=False):
    return {"op": "grouped", "mode": mode, "T": T, "E": E, "k": k, "K": K, "N": N, "pow2": pow2}


def _combine(T, E, k, D, *, train=True):
    return {"op": "combine", "T": T, "E": E, "k": k, "D": D, "train": train}


def _adamw(count, numel, *, param="bf16", grad="bf16", state="fp8"):
    return {"op": "adamw", "count": count, "numel": numel, "param": param, "grad": grad, "state": state}


def listed():
    return [
        # a decode batch's choice among many small experts: a launch or two
        {"name": "route_decode_16_tokens", **_route(16, 64, 6, dtype="bf16", train=False)},
        # the router of a training step, with padding tokens and masked experts, and its backward
        {"name": "route_train_16384_tokens", **_route(16384, 64, 6, renorm=False)},
        # one user's token through two of eight experts' up projections: the stream of two weights
        {"name": "grouped_decode_1_token", **_grouped("infer", 1, 8, 2, 4096, 14336)},
        # a decode batch over many small experts: six rows each on average, ragged, some experts without any
        {"name": "grouped_decode_64_tokens", **_grouped("infer", 64, 64, 6, 2048, 1408, pow2=True)},
        # a prompt of odd length through the down projections of eight experts
        {"name": "grouped_prompt_777_tokens", **_grouped("infer", 777, 8, 2, 14336, 4096)},
        # the forward of a training step, two of eight experts per token
        {"name": "grouped_fwd_8192_tokens", **_grouped("fwd", 8192, 8, 2, 4096, 14336)},
        # its two backward products: the largest case
        {"name": "grouped_bwd_8192_tokens", **_grouped("bwd", 8192, 8, 2, 4096, 14336)},
        # many small experts, an odd token count: groups of a hundred-odd rows each way
        {"name": "grouped_bwd_1531_tokens", **_grouped("bwd", 1531, 64, 6, 2048, 1408, pow2=True)},
        # a decode batch's outputs put together
        {"name": "combine_decode_64_tokens", **_combine(64, 64, 6, 2048, train=False)},
        # the same in a training step, forward and backward
        {"name": "combine_train_8192_tokens", **_combine(8192, 8, 2, 4096)},
        # a router's and norms' worth of small tensors, everything in 32 bits
        {"name": "adamw_small_fp32", **_adamw(150, 8192, param="fp32", grad="fp32", state="fp32")},
        # the weights of eight experts with their moments in 8 bits
        {"name": "adamw_experts_fp8", **_adamw(8, 4096 * 14336)},
    ]


def _cost(c):
    """A rough time of the plain form, in seconds."""
    w = work(c)
    if c["op"] == "grouped":
        return w["flops"] / 1e14 * 1.5 + w["bytes"] / 2e11
    return w["bytes"] / 2e11


def draw(rng):
    """One more case of the same ranges."""
    log = lambda lo, hi: math.exp(rng.uniform(math.log(lo), math.log(hi)))      # noqa: E731
    limit = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["route", "grouped", "grouped", "combine", "adamw"])
        E = int(log(4, 257))
        k = rng.randint(1, min(8, E))
        if op == "route":
            c = _route(int(log(1, 32769)), E, k, dtype=rng.choice(["bf16", "fp32"]), renorm=rng.random() < 0.5,
                       mask=rng.random() < 0.7, train=rng.random() < 0.6)
        elif op == "grouped":
            mode = rng.choice(["infer", "fwd", "bwd"])
            T = int(log(1, 1025)) if mode == "infer" else int(log(128, 16385))
            c = _grouped(mode, T, E, k, int(log(512, 14337)) // 16 * 16, int(log(512, 14337)) // 16 * 16, pow2=rng.random() < 0.3)
            if c["E"] * c["K"] * c["N"] > 8 * 4096 * 14336:
                continue
        elif op == "combine":
            c = _combine(int(log(1, 16385)), E, k, int(log(256, 8193)) // 8 * 8, train=rng.random() < 0.6)
        else:
            count = int(log(1, 200))
            c = _adamw(count, int(log(1000, 4e8)) // count + rng.randint(1, 99), param=rng.choice(["bf16", "fp32"]),
                       grad=rng.choice(["bf16", "fp32"]), state=rng.choice(["fp8", "fp32"]))
        if _cost(c) <= limit and max(c.get("K", 0) * c["T"] * k if op == "grouped" else 0, 1) <= 16384 * 14336:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def _randn(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen)


def _logits(gen, T, E, mask):
    """Router logits with popular and unpopular experts; mask: an expert that is out now and then, and padding tokens that
    have none."""
    x = _randn(gen, T, E) + 0.7 * _randn(gen, E)
    if mask:
        x = x.masked_fill(torch.rand((T, E), device="cuda", generator=gen) < 0.05, -math.inf)
        x = x.masked_fill(torch.rand((T, 1), device="cuda", generator=gen) < 0.02, -math.inf)
    return x


def _lists(experts, E, k):
    """Expert-ordered row lists of a choice [T, k] (-1: none): offsets [E + 1], row_token [T k], slot_row [T, k]."""
    key = torch.where(experts < 0, E, experts).reshape(-1).long()
    ordered, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(ordered, torch.arange(E + 1, device="cuda")).int()
    row_token = torch.where(ordered < E, order // k, -1).int()
    place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device="cuda"))
    return offsets, row_token, torch.where(key < E, place, -1).reshape(experts.shape).int()


def _routing(gen, T, E, k):
    """What a router hands to the products: expert-ordered rows of skewed groups, and a few padding tokens' rows at the end."""
    x = _logits(gen, T, E, False)
    experts = torch.topk(x, k, dim=1).indices
    if T > 256:
        experts = experts.masked_fill(torch.rand((T, 1), device="cuda", generator=gen) < 0.01, -1)
    return _lists(experts, E, k)


def _sizes(case):
    """Element counts of the tensors of a step: around the case's, odd ones among them."""
    n = case["numel"]
    return [max(1, n * (1 + 3 * i % 5) // 3 + 13 * i % 17) for i in range(case["count"])]


def _root_scale(amax):
    """The power-of-two scale of a block of moments."""
    s = (448.0 / amax.double().clamp(min=1e-12)).float()
    return (s.view(torch.int32) & -0x800000).view(torch.float32)


def _state_codes(x, roots):
    """Blocks [B, 256] of moments -> e4m3 codes and one scale each; of roots, what is not zero does not become zero."""
    s = _root_scale(x.abs().amax(1))
    y = x * s[:, None]
    if roots:
        y = torch.where(x > 0, y.clamp(min=2.0 ** -9), y)
    return y.to(E4M3), s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    if case["op"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        s["logits"] = _logits(gen, T, E, case["mask"]).to(DTYPES[case["dtype"]])
        if case["train"]:
            s["dgates"] = _randn(gen, T, k)
    elif case["op"] == "grouped":
        T, E, k, K, N = case["T"], case["E"], case["k"], case["K"], case["N"]
        s["offsets"], s["row_token"], _ = _routing(gen, T, E, k)
        s["most"] = max(1, int(s["offsets"].diff().max()))      # rows of the largest group: the plain form pads to it
        s["x"] = _randn(gen, T, K).to(torch.bfloat16)
        w = _randn(gen, E, N, K).mul_(0.02).to(torch.bfloat16)
        if case["mode"] == "infer":
            q, sw = _codes(w, 2, E4M3, case["pow2"])
            s["wq"], s["sw"] = q.to(E4M3).view(torch.uint8), sw.reshape(E, N)
        else:
            s["w"] = w
        if case["mode"] == "bwd":
            s["dy"] = _randn(gen, T * k, N).mul_(1e-3).to(torch.bfloat16)
    elif case["op"] == "combine":
        T, E, k, D = case["T"], case["E"], case["k"], case["D"]
        _, s["row_token"], s["slot_row"] = _routing(gen, T, E, k)
        s["y"] = _randn(gen, T * k, D).to(torch.bfloat16)
        s["gates"] = torch.softmax(_randn(gen, T, k), 1)
        if case["train"]:
            s["dout"] = _randn(gen, T, D).mul_(1e-3).to(torch.bfloat16)
    else:
        sizes = _sizes(case)
        B = STATE_BLOCK
        at, total = [], 0
        for n in sizes:      # the tensors are windows of flat buffers, each on a block boundary
            at.append(total)
            total += (n + B - 1) // B * B
        inside = torch.zeros(total, device="cuda")
        for a, n in zip(at, sizes):
            inside[a:a + n] = 1.0
        p = _randn(gen, total).mul_(0.02).mul_(inside)
        g = _randn(gen, total).mul_(1e-3).mul_(inside)
        m = _randn(gen, total).mul_(3e-4).mul_(inside)
        r = _randn(gen, total).abs_().mul_(1e-3).mul_(inside)
        quiet = (torch.rand(total // B, 1, device="cuda", generator=gen) > 0.03).float()      # rows that no token has used yet
        g.view(-1, B).mul_(quiet), m.view(-1, B).mul_(quiet), r.view(-1, B).mul_(quiet)
        s["p"], s["g"] = p.to(DTYPES[case["param"]]), g.to(DTYPES[case["grad"]])
        s["grad_scale"] = torch.full((1,), 0.75, device="cuda")      # what clipping has come to
        if case["state"] == "fp8":
            s["m"], s["sm"] = _state_codes(m.view(-1, B), False)
            s["v"], s["sv"] = _state_codes(r.view(-1, B), True)
            s["m"], s["v"] = s["m"].view(-1).view(torch.uint8), s["v"].view(-1).view(torch.uint8)
        else:
            s["m"], s["v"] = m, r.square_()
        window = lambda t, d=1: [t[a // d:a // d + (n + d - 1) // d] for a, n in zip(at, sizes)]      # noqa: E731
        s["windows"] = {name: window(s[name]) for name in ("p", "g", "m", "v")}
        if case["state"] == "fp8":
            s["windows"] |= {name: window(s[name], B) for name in ("sm", "sv")}
        if own:      # made once, where a program makes its parameters
            import paper_2507_16099_amd as fp8

            w = s["windows"]
            s["tensors"] = fp8.fp8_adamw_tensors(w["p"], w["g"], w["m"], w["v"], w.get("sm"), w.get("sv"))
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass


def _codes(x, dim, fmt, pow2):
    """x's codes (as the 32-bit values that they stand for) and scales with one scale per line along `dim`."""
    x = x.float()
    s = (FMAX[fmt] / x.abs().amax(dim, keepdim=True).double().clamp(min=1e-12)).float()
    if pow2:
        s = (s.view(torch.int32) & -0x800000).view(torch.float32)
    return (x * s).clamp(-FMAX[fmt], FMAX[fmt]).to(fmt).float(), s


def _plain_route(s):
    c, x = s["case"], s["logits"].float()
    E, k = c["E"], c["k"]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isfinite(top), top, 0.0))
    order = torch.sort(x, dim=1, descending=True, stable=True)
    chosen = order.values[:, :k] > -math.inf
    experts = torch.where(chosen, order.indices[:, :k], -1)
    picked = torch.where(chosen, e.gather(1, experts.clamp(min=0)), 0.0)
    total = (picked if c["renorm"] else e).sum(1, keepdim=True)
    total = torch.where(total > 0, total, 1.0)
    gates = picked / total
    offsets, row_token, slot_row = _lists(experts, E, k)
    out = {"gates": gates, "experts": experts.int(), "offsets": offsets, "row_token": row_token, "slot_row": slot_row}
    if c["train"]:
        inner = (s["dgates"] * gates).sum(1, keepdim=True)
        if c["renorm"]:
            own_part, d = gates * (s["dgates"] - inner), torch.zeros_like(x)
        else:
            own_part, d = gates * s["dgates"], -(e / total) * inner
        out["dlogits"] = d.scatter_add_(1, experts.clamp(min=0), torch.where(chosen, own_part, 0.0)).to(s["logits"].dtype)
    return out


def _plain_grouped(s):
    c, offsets, rows = s["case"], s["offsets"].long(), s["row_token"].long().clamp(min=0)
    pow2, M = c["pow2"], s["row_token"].numel()
    # rows padded to the largest group: [E, most], and the way back
    place = offsets[:-1, None] + torch.arange(s["most"], device="cuda")
    real = place < offsets[1:, None]
    place = torch.where(real, place, 0)
    row = torch.arange(M, device="cuda")
    group = torch.searchsorted(offsets[1:], row, right=True)
    there = (group < c["E"])[:, None]
    group = group.clamp(max=c["E"] - 1)
    inside = (row - offsets[group]).clamp(0, s["most"] - 1)
    padded = lambda v: torch.where(real[..., None], v[place], 0.0)                            # noqa: E731
    back = lambda v: torch.where(there, v[group, inside], 0.0).to(torch.bfloat16)             # noqa: E731
    if c["mode"] != "bwd":
        q, sx = _codes(s["x"], 1, E4M3, pow2)
        if c["mode"] == "infer":
            wq, sw = s["wq"].view(E4M3).float(), s["sw"][..., None]
        else:
            wq, sw = _codes(s["w"], 2, E4M3, pow2)
        y = torch.bmm(padded(q[rows]), wq.transpose(1, 2))
        return {"y": back(y * (1.0 / padded(sx[rows]).clamp(min=1e-30)) * (1.0 / sw.transpose(1, 2)))}
    g, sg = _codes(s["dy"], 1, E5M2, pow2)
    wq, sw = _codes(s["w"], 1, E4M3, pow2)
    dx = back(torch.bmm(padded(g), wq) * (1.0 / padded(sg).clamp(min=1e-30)) * (1.0 / sw))
    del g, wq
    g, sg = _codes(padded(s["dy"].float()), 1, E5M2, pow2)
    x, sx = _codes(padded(s["x"].float()[rows]), 1, E4M3, pow2)
    dw = torch.bmm(g.transpose(1, 2), x) * (1.0 / sg.transpose(1, 2)) * (1.0 / sx)
    return {"dx": dx, "dw": dw.to(torch.bfloat16)}


def _plain_combine(s):
    rows = s["slot_row"].long()
    taken = torch.where(rows[..., None] >= 0, s["y"][rows.clamp(min=0)].float(), 0.0)
    out = {"out": (taken * s["gates"][..., None]).sum(1).to(torch.bfloat16)}
    if s["case"]["train"]:
        d = s["dout"].float()[:, None, :]
        out["dgates"] = (taken * d).sum(2)
        spread = (d * s["gates"][..., None]).reshape(-1, s["case"]["D"])
        M = s["y"].shape[0]
        at = torch.where(rows >= 0, rows, M).reshape(-1)
        dy = torch.zeros((M + 1, s["case"]["D"]), device="cuda")
        dy[at] = spread
        out["dy"] = dy[:M].to(torch.bfloat16)
    return out


def _plain_adamw(s):
    h, fp8_state = HYPER, s["case"]["state"] == "fp8"
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).item()      # noqa: E731
    bc1, bc2 = 1 - h["beta1"] ** h["step"], 1 - h["beta2"] ** h["step"]
    decay, rate, inv_root = f32(1 - h["lr"] * h["weight_decay"]), f32(h["lr"] / bc1), f32(1 / math.sqrt(bc2))
    b1, c1, b2, c2 = f32(h["beta1"]), f32(1 - h["beta1"]), f32(h["beta2"]), f32(1 - h["beta2"])
    g = s["g"].float() * s["grad_scale"]
    if fp8_state:
        m = (s["m"].view(E4M3).float().view(-1, STATE_BLOCK) / s["sm"][:, None]).view(-1)
        r = (s["v"].view(E4M3).float().view(-1, STATE_BLOCK) / s["sv"][:, None]).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * c1
    v = v * b2 + (g * g) * c2
    r = torch.sqrt(v)
    p = s["p"].float() * decay - (m / (r * inv_root + f32(h["eps"]))) * rate
    s["p"].copy_(p)
    if not fp8_state:
        s["m"].copy_(m), s["v"].copy_(v)
        return {name: s[name] for name in ("p", "m", "v")}
    q, sm = _state_codes(m.view(-1, STATE_BLOCK), False)
    s["m"].view(E4M3).copy_(q.view(-1)), s["sm"].copy_(sm)
    q, sv = _state_codes(r.view(-1, STATE_BLOCK), True)
    s["v"].view(E4M3).copy_(q.view(-1)), s["sv"].copy_(sv)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    if s["case"]["state"] == "fp8":
        return {"p": s["p"], "m": s["m"].view(E4M3), "m_scale": s["sm"], "v_root": s["v"].view(E4M3), "v_scale": s["sv"]}
    return {name: s[name] for name in ("p", "m", "v")}


def _own_pass(s):
    import paper_2507_16099_amd as fp8

    c = s["case"]
    if c["op"] == "route":
        flags = fp8.FP8_ROUTE_RENORM if c["renorm"] else 0
        gates, experts, offsets, row_token, slot_row = fp8.fp8_moe_route(s["logits"], c["k"], flags)
        out = {"gates": gates, "experts": experts, "offsets": offsets, "row_token": row_token, "slot_row": slot_row}
        if c["train"]:
            out["dlogits"] = fp8.fp8_moe_route_bwd(s["dgates"], s["logits"], gates, experts, flags)
        return out
    if c["op"] == "grouped":
        flags = fp8.FP8_POW2_SCALE if c["pow2"] else 0
        if c["mode"] == "infer":
            return {"y": fp8.fp8_grouped_linear_fwd_prequantized(s["x"], s["wq"], fp8.FP8_E4M3FN, s["sw"], s["offsets"],
                                                                 fp8.FP8_E4M3FN, flags, row_token=s["row_token"])}
        recipe = fp8.Recipe(gran=fp8.FP8_ROW, flags=flags)
        if c["mode"] == "fwd":
            return {"y": fp8.fp8_grouped_linear_fwd(s["x"], s["w"], s["offsets"], recipe, row_token=s["row_token"])}
        dx, dw = fp8.fp8_grouped_linear_bwd(s["dy"], s["x"], s["w"], s["offsets"], recipe, row_token=s["row_token"])
        return {"dx": dx, "dw": dw}
    if c["op"] == "combine":
        out = {"out": fp8.fp8_moe_combine(s["y"], s["gates"], s["slot_row"])}
        if c["train"]:
            out["dy"], out["dgates"] = fp8.fp8_moe_combine_bwd(s["dout"], s["y"], s["gates"], s["slot_row"], s["row_token"])
        return out
    fp8.fp8_adamw_step(s["tensors"], grad_scale=s["grad_scale"], **HYPER)
    return _adamw_outputs(s)


def run(s):
    if own:
        return _own_pass(s)
    return {"route": _plain_route, "grouped": _plain_grouped, "combine": _plain_combine, "adamw": _plain_adamw}[s["case"]["op"]](s)


def work(case):
    op = case["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        b = T * E * (2 if case["dtype"] == "bf16" else 4)
        return {"bytes": b + 16.0 * T * k + 4 * E + (b * 2 + 12.0 * T * k if case["train"] else 0), "flops": 4.0 * T * E}
    if op == "grouped":
        T, E, k, K, N = case["T"], case["E"], case["k"], case["K"], case["N"]
        M = T * k
        if case["mode"] == "infer":      # experts that at least one token has chosen, were the choice even
            busy = E * (1 - (1 - k / E) ** T)
            return {"bytes": 2.0 * T * K + busy * N * (K + 4) + 2.0 * M * N, "flops": 2.0 * M * K * N}
        if case["mode"] == "fwd":
            return {"bytes": 2.0 * (T * K + E * N * K + M * N), "flops": 2.0 * M * K * N}
        return {"bytes": 2.0 * (M * N + T * K + E * N * K + M * K + E * N * K), "flops": 4.0 * M * K * N}
    if op == "combine":
        T, k, D = case["T"], case["k"], case["D"]
        b = 2.0 * T * k * D + 2.0 * T * D + 8.0 * T * k
        if case["train"]:      # dout and the outputs again, their gradients and the gates'
            b += 2.0 * T * D + 4.0 * T * k * D + 12.0 * T * k
        return {"bytes": b, "flops": (6.0 if case["train"] else 2.0) * T * k * D}
    n = float(sum(_sizes(case)))
    size = {"bf16": 2, "fp32": 4}
    state = 4.0 + 16.0 / STATE_BLOCK if case["state"] == "fp8" else 16.0
    return {"bytes": n * (2 * size[case["param"]] + size[case["grad"]] + state), "flops": 15.0 * n}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions


def _round_to(x, mantissa, least, most):
    """The nearest values with so many mantissa bits (ties to even), steps no finer than those at 2^least, saturating."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** least))).clamp(min=least)
    step = torch.exp2(e - mantissa)
    return (torch.round(x / step) * step).clamp(-most, most)


def _exact_values(x, dim, fmt, pow2):
    """What is left of x behind its codes, one scale per line along `dim`."""
    x = x.double()
    s = (FMAX[fmt] / x.abs().amax(dim, keepdim=True).clamp(min=1e-12)).float().double()
    if pow2:
        s = torch.exp2(torch.frexp(s)[1].double() - 1)
    scaled = (x * s).float().double()      # the product with the scale is rounded to 32 bits by definition
    return (_round_to(scaled, 3, -6, 448.0) if fmt is E4M3 else _round_to(scaled, 2, -14, 57344.0)) / s


def _exact_route(s):
    import numpy as np

    c, x = s["case"], s["logits"].double().cpu().numpy()
    T, E, k = c["T"], c["E"], c["k"]
    order = np.lexsort((np.broadcast_to(np.arange(E), (T, E)), -x), axis=1)[:, :k]
    value = np.take_along_axis(x, order, 1)
    chosen = value > -np.inf
    experts = np.where(chosen, order, -1)
    top = x.max(1, keepdims=True)
    e = np.exp(x - np.where(np.isfinite(top), top, 0.0))
    picked = np.where(chosen, np.take_along_axis(e, order, 1), 0.0)
    total = (picked if c["renorm"] else e).sum(1, keepdims=True)
    total = np.where(total > 0, total, 1.0)
    gates = picked / total
    flat = np.where(chosen, order, E).reshape(-1)
    by = np.argsort(flat, kind="stable")
    slot_row = np.empty(T * k, dtype=np.int64)
    slot_row[by] = np.arange(T * k)
    out = {"gates": gates, "experts": experts, "offsets": np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E + 1)[:E])]),
           "row_token": np.where(flat[by] < E, by // k, -1), "slot_row": np.where(flat < E, slot_row, -1).reshape(T, k)}
    if c["train"]:
        dg = s["dgates"].double().cpu().numpy()
        inner = (dg * gates).sum(1, keepdims=True)
        spread = np.zeros((T, E))
        np.put_along_axis(spread, order, np.where(chosen, dg, 0.0), 1)
        if c["renorm"]:
            share = np.zeros((T, E))
            np.put_along_axis(share, order, gates, 1)
            out["dlogits"] = share * (spread - inner)
        else:
            out["dlogits"] = e / total * (spread - inner)
    return {name: torch.from_numpy(np.ascontiguousarray(v)) for name, v in out.items()}


def _exact_grouped(s):
    c, offsets = s["case"], s["offsets"].tolist()
    rows, pow2, M = s["row_token"].long(), c["pow2"], s["row_token"].numel()
    K, N, f64 = c["K"], c["N"], dict(dtype=torch.float64, device="cuda")
    groups = [(e, slice(a, b)) for e, (a, b) in enumerate(zip(offsets, offsets[1:])) if b > a]
    if c["mode"] != "bwd":
        y, x = torch.zeros((M, N), **f64), _exact_values(s["x"], 1, E4M3, pow2)
        for e, at in groups:
            w = s["wq"][e].view(E4M3).double() / s["sw"][e].double()[:, None] if c["mode"] == "infer" else _exact_values(s["w"][e], 1, E4M3, pow2)
            y[at] = x[rows[at]] @ w.T
        return {"y": y}
    dx, dw, g = torch.zeros((M, K), **f64), torch.zeros((c["E"], N, K), **f64), _exact_values(s["dy"], 1, E5M2, pow2)
    for e, at in groups:
        dx[at] = g[at] @ _exact_values(s["w"][e], 0, E4M3, pow2)
        dw[e] = _exact_values(s["dy"][at], 0, E5M2, pow2).T @ _exact_values(s["x"][rows[at]], 0, E4M3, pow2)
    return {"dx": dx, "dw": dw}


def _exact_combine(s):
    M, D = s["y"].shape
    rows, gates = s["slot_row"].long(), s["gates"].double()
    y = torch.cat([s["y"].double(), torch.zeros((1, D), dtype=torch.float64, device="cuda")])      # no row: the zero one
    at = torch.where(rows >= 0, rows, M)
    total = torch.zeros((rows.shape[0], D), dtype=torch.float64, device="cuda")
    for j in range(rows.shape[1]):
        total += gates[:, j:j + 1] * y[at[:, j]]
    out = {"out": total}
    if s["case"]["train"]:
        d, dy = s["dout"].double(), torch.zeros_like(y)
        out["dgates"] = torch.empty_like(gates)
        for j in range(rows.shape[1]):
            out["dgates"][:, j] = (d * y[at[:, j]]).sum(1)
            dy[at[:, j]] = gates[:, j:j + 1] * d
        out["dy"] = dy[:M]
    return out


def _exact_adamw(s):
    h, B = HYPER, STATE_BLOCK
    g, p = s["g"].double() * s["grad_scale"].double(), s["p"].double()
    if s["case"]["state"] == "fp8":
        m = (s["m"].view(E4M3).double().view(-1, B) / s["sm"].double()[:, None]).reshape(-1)
        v = (s["v"].view(E4M3).double().view(-1, B) / s["sv"].double()[:, None]).reshape(-1).square()
    else:
        m, v = s["m"].double(), s["v"].double()
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    root = v.sqrt()
    step = m / (1 - h["beta1"] ** h["step"]) / (root / math.sqrt(1 - h["beta2"] ** h["step"]) + h["eps"])
    out = {"p": p - h["lr"] * h["weight_decay"] * p - h["lr"] * step}
    if s["case"]["state"] != "fp8":
        return out | {"m": m, "v": v}
    for name, x in (("m", m), ("v_root", root)):
        x = x.view(-1, B)
        scale = torch.exp2(torch.floor(torch.log2(448.0 / x.abs().amax(1).clamp(min=1e-12))))
        y = x * scale[:, None]
        if name == "v_root":
            y = torch.where(x > 0, y.clamp(min=2.0 ** -9), y)
        out[name] = _round_to(y, 3, -6, 448.0).reshape(-1)
        out[name.split("_")[0] + "_scale"] = scale
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "grouped": _exact_grouped, "combine": _exact_combine, "adamw": _exact_adamw}[case["op"]](s)
