"""What the operators around the FP8 products of a training step are measured on.

Four pieces of a step lie outside the block's FP8 products: the token embedding in front of them (forward, and the
gradient of the table), the layer norm between them (forward with the FP8 codes of the next product's operand, and its
backward pass), the router of the grouped products (experts, counts, order of the rows, balance and z losses, and the
gradient), and the clip of the gradients that the products leave (global norm, scaling).

``run`` computes them in plain torch operations in 32 bits (``own`` false) or through the package's entry points
(``own`` true); ``exact`` evaluates their definitions in 64 bits.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
DEVICE = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the package's smallest configuration (hidden 256) with one token more, from an FP32 master table: latency
        {"name": "embed_small", "op": "embed_fwd", "T": 257, "V": 50257, "D": 256, "fp32": True, "codes": False},
        # 8192 tokens of the 8B-class block (hidden 4096): the block's input and its FP8 codes under a delayed scale
        {"name": "embed_block_codes", "op": "embed_fwd", "T": 8192, "V": 131072, "D": 4096, "fp32": False, "codes": True},
        # gradient of that block's table, written whole (untouched rows are zeros)
        {"name": "embed_grad_block", "op": "embed_bwd", "T": 8192, "V": 131072, "D": 4096, "fp32": False, "accumulate": False},
        # gradient accumulated into an FP32 master gradient over micro-batches: only touched rows move
        {"name": "embed_grad_accumulate", "op": "embed_bwd", "T": 12345, "V": 50257, "D": 2048, "fp32": True, "accumulate": True},
        # norm of the smallest configuration, no residual: latency
        {"name": "norm_small", "op": "norm_fwd", "T": 256, "D": 256, "residual": False, "codes": False},
        # post-norm of the 8B-class block with its residual, and the codes of the next product's operand
        {"name": "norm_block_codes", "op": "norm_fwd", "T": 8192, "D": 4096, "residual": True, "codes": True},
        # its backward pass, and one of odd sizes
        {"name": "norm_grad_block", "op": "norm_bwd", "T": 8192, "D": 4096, "accumulate": False},
        {"name": "norm_grad_ragged", "op": "norm_bwd", "T": 4099, "D": 1032, "accumulate": True},
        # 8 experts, 2 active, 8192 tokens, FP32 logits: forward and backward of the router
        {"name": "route_8_experts", "op": "route", "T": 8192, "E": 8, "k": 2, "fp32": True, "normalize": True, "bias": True},
        # many small experts, BF16 logits with ties, masked experts and padded tokens, odd sizes
        {"name": "route_many_experts", "op": "route", "T": 16411, "E": 160, "k": 6, "fp32": False, "normalize": False, "bias": False},
        # every gradient of one 8B-class block: four BF16 weight gradients and its vectors into an FP32 bucket
        {"name": "clip_block", "op": "clip", "tensors": 8, "numel": 218103808, "fp32": False},
        # hundreds of FP32 gradients of odd sizes, most of them small: launches and tails count
        {"name": "clip_many", "op": "clip", "tensors": 389, "numel": 12345678, "fp32": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "norm_fwd", "norm_bwd", "route", "clip"])
    if op in ("embed_fwd", "embed_bwd"):
        c = {"op": op, "T": _log(rng, 1, 32768), "V": _log(rng, 2, 131072), "D": 8 * _log(rng, 1, 1024), "fp32": rng.random() < 0.5}
        while c["V"] * c["D"] > 131072 * 2048 or c["T"] * c["D"] > 8192 * 4096:
            c["D"] = 8 * max(1, c["D"] // 16)
        if op == "embed_fwd":
            c["codes"] = rng.random() < 0.5
        else:
            c["accumulate"] = rng.random() < 0.5
        return c
    if op in ("norm_fwd", "norm_bwd"):
        c = {"op": op, "T": _log(rng, 1, 65536), "D": 8 * _log(rng, 1, 2048)}
        while c["T"] * c["D"] > 8192 * 4096:
            c["T"] = max(1, c["T"] // 2)
        if op == "norm_fwd":
            c["residual"], c["codes"] = rng.random() < 0.5, rng.random() < 0.5
        else:
            c["accumulate"] = rng.random() < 0.5
        return c
    if op == "route":
        E = _log(rng, 2, 256)
        return {"op": op, "T": _log(rng, 1, 32768), "E": E, "k": rng.randint(1, min(E, 8)), "fp32": rng.random() < 0.5,
                "normalize": rng.random() < 0.5, "bias": rng.random() < 0.5}
    return {"op": op, "tensors": _log(rng, 1, 600), "numel": _log(rng, 1000, 100_000_000), "fp32": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 13)


def _normal(g, shape, std, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=dtype) * std


def _token_ids(g, T, V):
    """Token ids of a text: frequencies fall off with the rank (log-uniform ranks), the ranks lie anywhere in the table;
    one position in 64 is padding (-1)."""
    u = torch.rand(T, generator=g, device=DEVICE, dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    ids = torch.randperm(V, generator=g, device=DEVICE)[rank]
    pad = torch.rand(T, generator=g, device=DEVICE) < 1.0 / 64.0
    pad[0] = False
    return torch.where(pad, torch.full_like(ids, -1), ids)


def _clip_sizes(case):
    """Element counts of a model's gradients: for 8 tensors the projections of a block in their proportions, else a
    spread of sizes from vectors to matrices, odd ones among them; always `tensors` of them and about `numel` in all."""
    n, total = case["tensors"], case["numel"]
    if n == 8 and total == 218103808:
        return [6144 * 4096, 4096 * 4096, 28672 * 4096, 4096 * 14336, 4096, 4096, 128, 2]
    weight = [math.exp(4.0 * math.sin(1.7 * i + 0.3)) for i in range(n)]
    scale = total / sum(weight)
    return [max(1, int(w * scale)) for w in weight]


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = dict(case)
    f32 = torch.float32
    if op == "embed_fwd":
        T, V, D = case["T"], case["V"], case["D"]
        s["table"] = _normal(g, (V, D), 0.02, f32 if case["fp32"] else torch.bfloat16)
        s["ids"] = _token_ids(g, T, V)
        s["scale"] = 50.0                                    # 1 / 0.02: the inverse of the initialisation's deviation
        s["q_scale"] = torch.full((1,), 64.0, device=DEVICE)
        s["out"] = torch.empty((T, D), dtype=torch.bfloat16, device=DEVICE)
        s["out8"] = torch.empty((T, D), dtype=torch.uint8, device=DEVICE)
        s["amax"] = torch.empty(1, device=DEVICE)
    elif op == "embed_bwd":
        T, V, D = case["T"], case["V"], case["D"]
        dt = f32 if case["fp32"] else torch.bfloat16
        s["dy"] = _normal(g, (T, D), 1e-3)
        s["ids"] = _token_ids(g, T, V)
        s["scale"] = 50.0
        s["dtable"] = _normal(g, (V, D), 1e-2, dt) if case["accumulate"] else torch.empty((V, D), dtype=dt, device=DEVICE)
    elif op == "norm_fwd":
        T, D = case["T"], case["D"]
        col = torch.where(torch.rand(D, generator=g, device=DEVICE) < 0.01, 20.0, 1.0)      # a few outlier channels
        s["x"] = (torch.randn((T, D), generator=g, device=DEVICE) * col + 0.5).bfloat16()
        s["gamma"] = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEVICE)
        s["beta"] = 0.1 * torch.randn(D, generator=g, device=DEVICE)
        s["res"] = _normal(g, (T, D), 1.0) if case["residual"] else None
        s["eps"] = 1e-5
        s["q_scale"] = torch.full((1,), 16.0, device=DEVICE)
        s["out"] = torch.empty((T, D), dtype=torch.bfloat16, device=DEVICE)
        s["out8"] = torch.empty((T, D), dtype=torch.uint8, device=DEVICE)
        s["mean"], s["rstd"] = torch.empty(T, device=DEVICE), torch.empty(T, device=DEVICE)
        s["amax"] = torch.empty(1, device=DEVICE)
    elif op == "norm_bwd":
        T, D = case["T"], case["D"]
        x = (torch.randn((T, D), generator=g, device=DEVICE) + 0.5).bfloat16()
        s["x"] = x
        s["dout"] = _normal(g, (T, D), 1e-3)
        s["gamma"] = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEVICE)
        xd = x.double()
        mu = xd.mean(1)
        s["mean"] = mu.float()
        s["rstd"] = (1.0 / ((xd - mu[:, None]).square().mean(1) + 1e-5).sqrt()).float()
        s["dx"] = torch.empty_like(x)
        fill = torch.randn if case["accumulate"] else torch.zeros
        extra = {"generator": g} if case["accumulate"] else {}
        s["dgamma"], s["dbeta"] = fill(D, device=DEVICE, **extra), fill(D, device=DEVICE, **extra)
    elif op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        skew = torch.randn(E, generator=g, device=DEVICE)                                   # some experts are liked more
        logits = torch.randn((T, E), generator=g, device=DEVICE) * 1.5 + skew
        logits = logits if case["fp32"] else logits.bfloat16()
        if E > 8:                                            # experts that a token may not use, and padded tokens
            logits[torch.rand((T, E), generator=g, device=DEVICE) < 0.02] = -math.inf
            pad = torch.rand(T, generator=g, device=DEVICE) < 0.01
            pad[0] = False
            logits[pad] = -math.inf
            logits[0, 0] = 1.0
        s["logits"] = logits
        s["bias"] = 0.2 * torch.randn(E, generator=g, device=DEVICE) if case["bias"] else None
        s["balance_coef"], s["z_coef"] = 0.01, 0.001
        s["dloss"] = torch.ones(1, device=DEVICE)
        s["dweight"] = 1e-4 * torch.randn((T, k), generator=g, device=DEVICE)
        i32 = {"dtype": torch.int32, "device": DEVICE}
        s["expert"], s["weight"] = torch.empty((T, k), **i32), torch.empty((T, k), device=DEVICE)
        s["counts"], s["offsets"] = torch.empty(E, **i32), torch.empty(E + 1, **i32)
        s["rows"], s["n_routed"] = torch.empty(T * k, **i32), torch.empty(1, **i32)
        s["loss"] = torch.empty(2, device=DEVICE)
        s["dlogits"] = torch.empty_like(logits)
    else:
        sizes = _clip_sizes(case)
        dt = f32 if case["fp32"] else torch.bfloat16
        s["grads"] = [_normal(g, (n,), 1e-3 * (1 + i % 5), dt) for i, n in enumerate(sizes)]
        starts, at = [], 0
        for n in sizes:                                      # the optimizer's flat bucket: every tensor on 16 bytes
            starts.append(at)
            at += -(-n // 8) * 8
        s["bucket"] = torch.zeros(at, device=DEVICE)
        s["outs"] = [s["bucket"][a:a + n] for a, n in zip(starts, sizes)]
        s["gaps"] = [torch.zeros(-n % 8, dtype=dt, device=DEVICE) for n in sizes]
        s["max_norm"] = 1.0
        s["norm"] = torch.empty(1, device=DEVICE)
    return s


def work(case):
    op = case["op"]
    if op == "embed_fwd":
        T, D = case["T"], case["D"]
        rows = min(T, case["V"])                             # at most: tokens that repeat share their row
        return {"bytes": 8 * T + rows * D * (4 if case["fp32"] else 2) + T * D * (3 if case["codes"] else 2), "flops": T * D}
    if op == "embed_bwd":
        T, V, D, b = case["T"], case["V"], case["D"], 4 if case["fp32"] else 2
        moved = 2 * min(T, V) if case["accumulate"] else V
        return {"bytes": 8 * T + 2 * T * D + moved * D * b, "flops": 2 * T * D}
    if op == "norm_fwd":
        T, D = case["T"], case["D"]
        return {"bytes": T * D * (4 + 2 * case["residual"] + case["codes"]) + 8 * D + 8 * T, "flops": 8 * T * D}
    if op == "norm_bwd":
        T, D = case["T"], case["D"]
        return {"bytes": 6 * T * D + 4 * D * (3 + 2 * case["accumulate"]) + 8 * T, "flops": 14 * T * D}
    if op == "route":
        T, E, k, b = case["T"], case["E"], case["k"], 4 if case["fp32"] else 2
        return {"bytes": 3 * T * E * b + T * k * (4 + 4 + 4 + 8), "flops": 20 * T * E}
    n = sum(_clip_sizes(case))
    return {"bytes": n * (2 * (4 if case["fp32"] else 2) + 4), "flops": 3 * n}


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"embed_fwd": _embed_fwd, "embed_bwd": _embed_bwd, "norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd,
            "route": _route, "clip": _clip}[s["op"]](s)


def _codes(values_bf16, q_scale):
    v = (values_bf16.float() * q_scale).clamp(-E4M3_MAX, E4M3_MAX)
    return v.to(torch.float8_e4m3fn)


def _embed_fwd(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if s["codes"]:
            fp8.fp8_embedding_fwd_q(s["table"], s["ids"], s["scale"], s["q_scale"], fp8.E4M3, s["out"], s["out8"], s["amax"])
            return {"out": s["out"], "codes": s["out8"].view(torch.float8_e4m3fn), "amax": s["amax"]}
        fp8.fp8_embedding_fwd(s["table"], s["ids"], s["scale"], s["out"], s["amax"])
        return {"out": s["out"], "amax": s["amax"]}
    ids, V = s["ids"], s["V"]
    there = (ids >= 0) & (ids < V)
    rows = s["table"][ids.clamp(0, V - 1)].float() * s["scale"]
    out = torch.where(there[:, None], rows, torch.zeros_like(rows)).bfloat16()
    got = {"out": out, "amax": out.abs().max().float().reshape(1)}
    if s["codes"]:
        got["codes"] = _codes(out, s["q_scale"])
    return got


def _embed_bwd(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if "ws" not in s:
            s["ws"] = torch.empty(fp8.fp8_embedding_bwd_workspace_bytes(s["T"], s["V"], s["D"]), dtype=torch.uint8, device=DEVICE)
        fp8.fp8_embedding_bwd(s["dy"], s["ids"], s["scale"], s["dtable"], s["ws"], accumulate=s["accumulate"])
        return {"dtable": s["dtable"]}
    ids, V = s["ids"], s["V"]
    there = (ids >= 0) & (ids < V)
    dy = torch.where(there[:, None], s["dy"].float(), 0.0)
    grad = torch.zeros((V, s["D"]), device=DEVICE)
    grad.index_add_(0, ids.clamp(0, V - 1), dy)
    grad.mul_(s["scale"])
    if s["accumulate"]:
        s["dtable"].copy_(s["dtable"].float() + grad)
        return {"dtable": s["dtable"]}
    return {"dtable": grad.to(s["dtable"].dtype)}


def _norm_fwd(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if s["codes"]:
            fp8.fp8_layernorm_fwd_q(s["x"], s["gamma"], s["beta"], s["eps"], s["q_scale"], fp8.E4M3, s["out"], s["out8"],
                                    mean=s["mean"], rstd=s["rstd"], residual=s["res"], amax_out=s["amax"])
            return {"out": s["out"], "mean": s["mean"], "rstd": s["rstd"], "codes": s["out8"].view(torch.float8_e4m3fn),
                    "amax": s["amax"]}
        fp8.fp8_layernorm_fwd(s["x"], s["gamma"], s["beta"], s["eps"], s["out"], mean=s["mean"], rstd=s["rstd"],
                              residual=s["res"], amax_out=s["amax"])
        return {"out": s["out"], "mean": s["mean"], "rstd": s["rstd"], "amax": s["amax"]}
    x = s["x"].float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / (c.square().mean(1) + s["eps"]).sqrt()
    y = c * rstd[:, None] * s["gamma"] + s["beta"]
    if s["res"] is not None:
        y = y + s["res"].float()
    out = y.bfloat16()
    got = {"out": out, "mean": mean, "rstd": rstd, "amax": out.abs().max().float().reshape(1)}
    if s["codes"]:
        got["codes"] = _codes(out, s["q_scale"])
    return got


def _norm_bwd(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if "ws" not in s:
            s["ws"] = torch.empty(fp8.fp8_layernorm_bwd_workspace_bytes(s["T"], s["D"]), dtype=torch.uint8, device=DEVICE)
        fp8.fp8_layernorm_bwd(s["dout"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"],
                              accumulate=s["accumulate"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    dout, rstd = s["dout"].float(), s["rstd"][:, None]
    xhat = (s["x"].float() - s["mean"][:, None]) * rstd
    g = dout * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    dgamma, dbeta = (dout * xhat).sum(0), dout.sum(0)
    if s["accumulate"]:
        s["dgamma"] += dgamma
        s["dbeta"] += dbeta
        dgamma, dbeta = s["dgamma"], s["dbeta"]
    return {"dx": dx.bfloat16(), "dgamma": dgamma, "dbeta": dbeta}


def _route(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if "ws" not in s:
            s["ws"] = torch.empty(fp8.fp8_moe_route_workspace_bytes(s["T"], s["E"]), dtype=torch.uint8, device=DEVICE)
        fp8.fp8_moe_route(s["logits"], s["bias"], s["normalize"], s["balance_coef"], s["z_coef"], s["expert"], s["weight"],
                          s["counts"], s["offsets"], s["rows"], s["n_routed"], s["loss"], s["ws"])
        fp8.fp8_moe_route_bwd(s["logits"], s["expert"], s["counts"], s["n_routed"], s["normalize"], s["balance_coef"],
                              s["z_coef"], s["dloss"], s["dweight"], s["dlogits"])
        return {"expert": s["expert"], "weight": s["weight"], "counts": s["counts"], "offsets": s["offsets"],
                "rows": s["rows"], "n_routed": s["n_routed"], "loss": s["loss"], "dlogits": s["dlogits"]}
    T, E, k = s["T"], s["E"], s["k"]
    l = s["logits"].float()
    routed = (l > -math.inf).any(1)
    top = torch.where(routed, l.max(1).values, 0.0)
    e = torch.exp(l - top[:, None])
    total = torch.where(routed, e.sum(1), 1.0)
    p = e / total[:, None]
    lse = torch.where(routed, top + torch.log(total), 0.0)
    score = l if s["bias"] is None else l + s["bias"]
    value, order = torch.sort(score, dim=1, descending=True, stable=True)       # ties: the lowest expert first
    chosen = value[:, :k] > -math.inf
    index = order[:, :k]
    if s["normalize"]:
        picked = torch.where(chosen, l.gather(1, index), -math.inf)
        high = torch.where(routed, picked.max(1).values, 0.0)
        w = torch.exp(picked - high[:, None])
        w = w / torch.where(routed, w.sum(1), 1.0)[:, None]
    else:
        w = torch.where(chosen, p.gather(1, index), 0.0)
    expert = torch.where(chosen, index, -1).int()
    key = torch.where(chosen, index, E).reshape(-1)
    counts = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE).index_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), counts.cumsum(0)])
    by_expert, flat = torch.sort(key, stable=True)
    rows = torch.where(by_expert < E, flat, -1).int()
    n = routed.sum().float()
    share = counts.float() * E / (n * k)
    loss = torch.stack([s["balance_coef"] * (share * (p.sum(0) / n)).sum(), s["z_coef"] * lse.square().sum() / n])
    # gradient
    d = s["dloss"]
    dw = torch.where(chosen, s["dweight"], 0.0)
    u = (d * s["balance_coef"] * share / n).expand(T, E)
    if not s["normalize"]:
        u = u.scatter_add(1, index, dw)
    dl = p * (u - (u * p).sum(1, keepdim=True)) + (d * s["z_coef"] * 2.0 / n) * lse[:, None] * p
    if s["normalize"]:
        dl = dl.scatter_add(1, index, w * (dw - (dw * w).sum(1, keepdim=True)))
    return {"expert": expert, "weight": w, "counts": counts.int(), "offsets": offsets.int(), "rows": rows,
            "n_routed": n.int().reshape(1), "loss": loss, "dlogits": dl.to(s["logits"].dtype)}


def _clip(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if "items" not in s:
            s["items"] = fp8.fp8_grad_items(s["grads"], s["outs"])
            s["ws"] = torch.empty(fp8.fp8_grad_norm_workspace_bytes(s["items"]), dtype=torch.uint8, device=DEVICE)
        fp8.fp8_grad_norm(s["items"], s["norm"], s["ws"])
        fp8.fp8_grad_clip(s["items"], s["norm"], s["max_norm"])
        return {"norm": s["norm"], "bucket": s["bucket"]}
    flat = torch.cat([x for pair in zip(s["grads"], s["gaps"]) for x in pair]).float()
    norm = flat.square().sum().sqrt()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return {"norm": norm.reshape(1), "bucket": flat * factor}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s, op, f64 = prepare(case, seed), case["op"], torch.float64
    if op == "embed_fwd":
        padded = torch.cat([s["table"], s["table"].new_zeros((1, case["D"]))])              # id -1 reads the row of zeros
        out = padded[s["ids"]].double() * s["scale"]
        codes = (out * s["q_scale"].double()).clamp(-E4M3_MAX, E4M3_MAX) if case["codes"] else None
        return {"out": out, "codes": codes, "amax": None}
    if op == "embed_bwd":
        keep = s["ids"] >= 0
        base = s["dtable"].double() if case["accumulate"] else torch.zeros(s["dtable"].shape, dtype=f64, device=DEVICE)
        base.index_put_((s["ids"][keep],), s["dy"][keep].double() * s["scale"], accumulate=True)
        return {"dtable": base}
    if op == "norm_fwd":
        x = s["x"].double()
        mean = x.sum(1) / case["D"]
        var = x.square().sum(1) / case["D"] - mean * mean
        rstd = (var + s["eps"]) ** -0.5
        out = (x - mean.unsqueeze(1)) * (rstd.unsqueeze(1) * s["gamma"].double()) + s["beta"].double()
        if case["residual"]:
            out += s["res"].double()
        codes = (out * s["q_scale"].double()).clamp(-E4M3_MAX, E4M3_MAX) if case["codes"] else None
        return {"out": out, "mean": mean, "rstd": rstd, "codes": codes, "amax": None}
    if op == "norm_bwd":
        with torch.enable_grad():
            x = s["x"].double().requires_grad_()
            gamma, beta = s["gamma"].double().requires_grad_(), torch.zeros(case["D"], dtype=f64, device=DEVICE, requires_grad=True)
            c = x - x.mean(1, keepdim=True)
            y = c * (c.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gamma + beta
            dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dout"].double())
        if case["accumulate"]:
            dgamma, dbeta = dgamma + s["dgamma"].double(), dbeta + s["dbeta"].double()
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        score = s["logits"].float() if s["bias"] is None else s["logits"].float() + s["bias"]
        order = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :k]
        open_ = score.gather(1, order) > -math.inf
        live = open_.any(1)
        hot = torch.zeros((T, E), dtype=f64, device=DEVICE).scatter_(1, order, open_.double())
        share = hot.sum(0) * E / (live.sum() * k)
        with torch.enable_grad():
            l = s["logits"].double().requires_grad_()
            ll = l[live]
            logp = torch.log_softmax(ll, 1)
            lse = torch.logsumexp(ll, 1)
            loss = torch.stack([s["balance_coef"] * (share * logp.exp().mean(0)).sum(), s["z_coef"] * lse.square().mean()])
            at, ok = order[live], open_[live]
            if case["normalize"]:
                part = torch.softmax(ll.gather(1, at).masked_fill(~ok, -math.inf), 1)
            else:
                part = logp.gather(1, at).exp() * ok
            dl, = torch.autograd.grad(loss.sum() + (part * torch.where(ok, s["dweight"][live].double(), 0.0)).sum(), l)
        weight = torch.zeros((T, k), dtype=f64, device=DEVICE)
        weight[live] = part.detach()
        return {"expert": None, "weight": weight, "counts": None, "offsets": None, "rows": None, "n_routed": None,
                "loss": loss.detach(), "dlogits": torch.nan_to_num(dl)}
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(x, dtype=f64)) ** 2 for x in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + 1e-6))
    bucket = torch.zeros(s["bucket"].numel(), dtype=f64, device=DEVICE)
    for x, out in zip(s["grads"], s["outs"]):
        at = out.storage_offset()
        bucket[at:at + x.numel()] = x.double() * factor
    return {"norm": torch.tensor([norm], dtype=f64), "bucket": bucket}
