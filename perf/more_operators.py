"""What the operators between a block's FP8 products are measured on, and the optimizer behind them.

Rotary positions on the fused QKV projection (its table, forward with the attention's FP8 codes, gradient), the joint of two
blocks (norm behind a block, gate, residual scale, norm in front of the next one; forward with the FP8 codes, gradient), and
AdamW over many tensors (clip, step, BF16 copy and FP8 codes of the weights; states of 32 or of 8 bits).

``run`` computes them in plain torch operations in 32 bits (``own`` false) or through the package's entry points
(``own`` true); ``exact`` evaluates their definitions in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
E4M3_MAX, E5M2_MAX = 448.0, 57344.0
ALPHA = 0.7                                                   # of the tanh regulariser
BLOCK = 128                                                   # values that share a scale in the optimizer's 8-bit states


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # table of a 131072-token context, scaled by parts from one of 8192: every training job builds it
        {"name": "rope_table_long", "op": "table", "N": 131072, "rot": 128, "scaling": "parts"},
        # a few new tokens at positions of their own, heads of the 8B-class block: latency
        {"name": "rope_tokens", "op": "rope_fwd", "T": 3, "Hq": 32, "Hkv": 8, "d": 128, "rot": 128, "N": 131072, "mode": "rms",
         "interleaved": False, "positions": True, "codes": True},
        # 8192 tokens of the 8B-class block: QK norm, rotation, FP8 codes of Q, K and V for the attention
        {"name": "rope_block_codes", "op": "rope_fwd", "T": 8192, "Hq": 32, "Hkv": 8, "d": 128, "rot": 128, "N": 4096, "mode": "rms",
         "interleaved": False, "positions": False, "codes": True},
        # a packed batch of odd length with padding, interleaved pairs on half of each head, BF16 results
        {"name": "rope_ragged", "op": "rope_fwd", "T": 5003, "Hq": 12, "Hkv": 12, "d": 64, "rot": 32, "N": 2048, "mode": "none",
         "interleaved": True, "positions": True, "codes": False},
        # gradient of the block's QKV projection as the E5M2 operand of its products
        {"name": "rope_grad_block", "op": "rope_bwd", "T": 8192, "Hq": 32, "Hkv": 8, "d": 128, "rot": 128, "N": 4096, "mode": "rms",
         "interleaved": False, "positions": False, "codes": True},
        # the smallest configuration's joint (hidden 256), a token over: latency
        {"name": "norm_small", "op": "norm_fwd", "T": 257, "D": 256, "post": "rms", "gate": "none", "pre": True, "codes": True},
        # 8B-class block: norm behind the block, residual, norm in front of the next, codes of the next product's operand
        {"name": "norm_block_codes", "op": "norm_fwd", "T": 8192, "D": 4096, "post": "rms", "gate": "none", "pre": True, "codes": True},
        # its gradient with a gate per token and channel, E5M2 codes of the block's output gradient
        {"name": "norm_grad_block", "op": "norm_bwd", "T": 8192, "D": 4096, "post": "rms", "gate": "sigmoid", "pre": True, "dh": True,
         "codes": True, "accumulate": False},
        # odd sizes, a scale per channel in place of the norm, gradients of the scales added to
        {"name": "norm_grad_ragged", "op": "norm_bwd", "T": 4099, "D": 1032, "post": "scale", "gate": "none", "pre": True, "dh": True,
         "codes": False, "accumulate": True},
        # the weights of one 8B-class block: FP32 states, clip, BF16 copy and FP8 codes for the next step
        {"name": "adamw_block", "op": "adamw", "tensors": 8, "numel": 218103808, "fp32": False, "bits": 32, "codes": True},
        # the same with states of 8 bits
        {"name": "adamw_block_8bit", "op": "adamw", "tensors": 8, "numel": 218103808, "fp32": False, "bits": 8, "codes": True},
        # hundreds of tensors of odd sizes, FP32 gradients, most of them small: launches and tails count
        {"name": "adamw_many_8bit", "op": "adamw", "tensors": 389, "numel": 12345678, "fp32": True, "bits": 8, "codes": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["table", "rope_fwd", "rope_bwd", "norm_fwd", "norm_bwd", "adamw"])
    flip = lambda: rng.random() < 0.5  # noqa: E731
    if op == "table":
        return {"op": op, "N": _log(rng, 1, 131072), "rot": 16 * rng.randint(1, 8),
                "scaling": rng.choice(["plain", "linear", "ntk", "parts"])}
    if op in ("rope_fwd", "rope_bwd"):
        d = rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256])
        Hkv = _log(rng, 1, 16)
        c = {"op": op, "T": _log(rng, 1, 32768), "Hq": Hkv * _log(rng, 1, 8), "Hkv": Hkv, "d": d,
             "rot": d if flip() else 16 * rng.randint(1, d // 16), "N": _log(rng, 16, 32768), "mode": rng.choice(["rms", "tanh", "none"]),
             "interleaved": flip(), "positions": flip(), "codes": flip()}
        while c["T"] * (c["Hq"] + 2 * Hkv) * d > 8192 * 6144:
            c["T"] = max(1, c["T"] // 2)
        return c
    if op in ("norm_fwd", "norm_bwd"):
        c = {"op": op, "T": _log(rng, 1, 65536), "D": 8 * _log(rng, 1, 2048), "post": rng.choice(["rms", "scale", "none"]),
             "gate": rng.choice(["none", "linear", "sigmoid"]), "pre": flip(), "codes": flip()}
        while c["T"] * c["D"] > 8192 * 4096:
            c["T"] = max(1, c["T"] // 2)
        if op == "norm_bwd":
            c["dh"], c["accumulate"] = flip() or not c["pre"], flip()
        return c
    return {"op": op, "tensors": _log(rng, 1, 600), "numel": _log(rng, 1000, 100_000_000), "fp32": flip(),
            "bits": rng.choice([8, 32]), "codes": flip()}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 29)


def _normal(g, shape, std, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device=DEVICE) * std).to(dtype)


def _outlier_columns(g, D):
    return torch.where(torch.rand(D, generator=g, device=DEVICE) < 0.01, 20.0, 1.0)


SCALING = {"factor": 16.0, "original_len": 8192.0, "turns_low": 1.0, "turns_high": 32.0}


def _magnitude(scaling):
    return 1.0 + 0.1 * math.log(SCALING["factor"]) if scaling == "parts" else 1.0


def _turns(rot, scaling, base):
    """Turns per position of each pair, in 64 bits."""
    i = torch.arange(rot // 2, device=DEVICE, dtype=torch.float64)
    factor = SCALING["factor"]
    if scaling == "ntk" and rot > 2:
        base = base * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        n = SCALING["original_len"] * f / (2.0 * math.pi)
        w = ((n - SCALING["turns_low"]) / (SCALING["turns_high"] - SCALING["turns_low"])).clamp(0.0, 1.0)
        f = (1.0 - w) * f / factor + w * f
    return f / (2.0 * math.pi)


def _positions(g, T, N):
    """A packed batch: stretches that count on from anywhere in the context, one position in 64 is padding."""
    starts = torch.randint(0, N, (T // 100 + 1,), generator=g, device=DEVICE)
    t = torch.arange(T, device=DEVICE)
    pos = (starts[t // 100] + t % 100) % N
    pad = torch.rand(T, generator=g, device=DEVICE) < 1.0 / 64.0
    pad[0] = False
    return torch.where(pad, torch.full_like(pos, -1), pos)


def _sizes(case):
    """Element counts of a model's weights: for 8 tensors the projections of a block in their proportions, else a spread of
    sizes from vectors to matrices, odd ones among them; always `tensors` of them and about `numel` in all."""
    n, total = case["tensors"], case["numel"]
    if n == 8 and total == 218103808:
        return [6144 * 4096, 4096 * 4096, 28672 * 4096, 4096 * 14336, 4096, 4096, 128, 2]
    weight = [math.exp(4.0 * math.sin(1.7 * i + 0.3)) for i in range(n)]
    scale = total / sum(weight)
    return [max(1, int(w * scale)) for w in weight]


def _block_exponent(a):
    """Biased exponents e of the smallest powers of two with a <= 448 * 2^(e - 127), from the bits of `a` (FP32, >= 0)."""
    return (((a.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=1)


def _power(e):
    return (e.to(torch.int32) << 23).view(torch.float32)


def _encode_nearest(x):
    x = x.reshape(-1, BLOCK)
    e = _block_exponent(x.abs().amax(1))
    return (x * _power(254 - e)[:, None]).to(torch.float8_e4m3fn).reshape(-1).view(torch.uint8), e.to(torch.uint8)


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = dict(case)
    f32, bf16, u8 = torch.float32, torch.bfloat16, torch.uint8
    empty = lambda *shape, dtype=bf16: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
    if op == "table":
        s["base"] = 10.0 ** (4.0 + 2.0 * float(torch.rand(1, generator=g, device=DEVICE)))
        s["cos"], s["sin"] = empty(case["N"], case["rot"] // 2, dtype=f32), empty(case["N"], case["rot"] // 2, dtype=f32)
    elif op in ("rope_fwd", "rope_bwd"):
        T, Hq, Hkv, d = case["T"], case["Hq"], case["Hkv"], case["d"]
        W = (Hq + 2 * Hkv) * d
        angle = torch.arange(case["N"], device=DEVICE, dtype=torch.float64)[:, None] * _turns(case["rot"], "plain", 500000.0) * (2.0 * math.pi)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["pos"] = _positions(g, T, case["N"]).to(torch.int32 if seed % 2 else torch.int64) if case["positions"] else None
        s["qkv"] = (torch.randn((T, W), generator=g, device=DEVICE) * _outlier_columns(g, W)).to(bf16)
        s["eps"] = 1e-6
        if op == "rope_fwd":
            for n, H in (("q", Hq), ("k", Hkv), ("v", Hkv)):
                s[n] = empty(T, H, d, dtype=u8 if case["codes"] else bf16)
            s["scales"] = torch.tensor([32.0, 16.0, 8.0], device=DEVICE)
            s["amax"] = empty(3, dtype=f32)
        else:
            s["dq"], s["dk"], s["dv"] = _normal(g, (T, Hq, d), 1e-3), _normal(g, (T, Hkv, d), 2e-3), _normal(g, (T, Hkv, d), 1e-3)
            s["scale"] = torch.full((1,), 2.0 ** 20, device=DEVICE)
            s["dqkv"] = empty(T, W, dtype=u8 if case["codes"] else bf16)
            s["amax"] = empty(1, dtype=f32)
    elif op in ("norm_fwd", "norm_bwd"):
        T, D = case["T"], case["D"]
        y = (torch.randn((T, D), generator=g, device=DEVICE) * _outlier_columns(g, D)).to(bf16)
        x = _normal(g, (T, D), 1.0)
        gate = _normal(g, (T, D), 1.0) if case["gate"] != "none" else None
        gamma_post = 0.5 + 0.1 * torch.randn(D, generator=g, device=DEVICE) if case["post"] != "none" else None
        gamma_pre = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEVICE) if case["pre"] else None
        s |= {"y": y, "gate_in": gate, "gamma_post": gamma_post, "gamma_pre": gamma_pre, "a": 0.9, "b": 0.7, "eps": 1e-5}
        s["r_post"] = empty(T, dtype=f32) if case["post"] == "rms" else None
        s["r_pre"] = empty(T, dtype=f32) if case["pre"] else None
        if op == "norm_fwd":
            s["x"], s["h"], s["amax"] = x, empty(T, D), empty(1, dtype=f32)
            s["out"] = empty(T, D) if case["pre"] and not case["codes"] else None
            s["out8"] = empty(T, D, dtype=u8) if case["codes"] else None
            s["scale"] = torch.full((1,), 16.0, device=DEVICE)
        else:
            yf = y.float()
            z = yf
            if case["post"] == "rms":
                s["r_post"] = 1.0 / (yf.square().mean(1) + s["eps"]).sqrt()
                z = yf * s["r_post"][:, None]
            if gamma_post is not None:
                z = z * gamma_post
            if gate is not None:
                z = z * (torch.sigmoid(gate.float()) if case["gate"] == "sigmoid" else gate.float())
            s["h"] = (s["a"] * x.float() + s["b"] * z).to(bf16)
            if case["pre"]:
                s["r_pre"] = 1.0 / (s["h"].float().square().mean(1) + s["eps"]).sqrt()
            s["dout"] = _normal(g, (T, D), 1e-3) if case["pre"] else None
            s["dh"] = _normal(g, (T, D), 1e-3) if case["dh"] else None
            s["dx"], s["dy"] = empty(T, D), empty(T, D, dtype=u8 if case["codes"] else bf16)
            s["dgate"] = empty(T, D) if gate is not None else None
            s["scale"], s["amax"] = torch.full((1,), 2.0 ** 20, device=DEVICE), empty(1, dtype=f32)
            for n, there in (("dgamma_post", gamma_post is not None), ("dgamma_pre", case["pre"])):
                s[n] = torch.randn(D, generator=g, device=DEVICE) * 0.1 if there else None
    else:
        sizes = _sizes(case)
        dt = f32 if case["fp32"] else bf16
        padded = [-(-n // BLOCK) * BLOCK for n in sizes]
        starts = [0]
        for n in padded:
            starts.append(starts[-1] + n)
        total = starts.pop()
        s["grads"] = [_normal(g, (n,), 1e-3 * (1 + i % 5), dt) for i, n in enumerate(sizes)]
        s["gaps"] = [torch.zeros(p - n, dtype=dt, device=DEVICE) for n, p in zip(sizes, padded)]
        s["counts"] = torch.tensor(padded, device=DEVICE)
        s["starts"] = torch.tensor(starts, device=DEVICE)
        live = torch.ones(total, device=DEVICE, dtype=torch.bool)
        for a, n, p in zip(starts, sizes, padded):
            live[a + n:a + p] = False
        p0 = torch.where(live, torch.randn(total, generator=g, device=DEVICE) * 0.02, 0.0)
        m0 = torch.where(live, torch.randn(total, generator=g, device=DEVICE) * 3e-4, 0.0)
        r0 = torch.where(live, torch.rand(total, generator=g, device=DEVICE) * 2e-3 + 1e-4, 0.0)
        s["p"] = p0
        if case["bits"] == 8:
            s["m"], s["me"] = _encode_nearest(m0)
            s["v"], s["ve"] = _encode_nearest(r0)
        else:
            s["m"], s["v"], s["me"], s["ve"] = m0, r0.square(), None, None
        s["p16"] = p0.to(bf16)
        s["p8"] = torch.zeros(total, dtype=u8, device=DEVICE) if case["codes"] else None
        s["q_scale"] = 1024.0 + 1024.0 * torch.rand(len(sizes), generator=g, device=DEVICE)
        s["amax"] = empty(len(sizes), dtype=f32)
        s["decay"] = [0.0 if n < 5000 else 0.1 for n in sizes]
        s["decays"] = torch.tensor(s["decay"], device=DEVICE)
        s["lr"] = torch.full((1,), 3e-4, device=DEVICE)
        s["step"] = torch.full((1,), 100, dtype=torch.int32, device=DEVICE)
        s["norm"] = torch.full((1,), 2.5, device=DEVICE)
        s["seed"] = 0x1234567890ABCDEF
        s |= {"beta1": 0.9, "beta2": 0.95, "adam_eps": 1e-8, "max_norm": 1.0}
        cut = lambda t, k=1: [t[a // k:a // k + -(-n // k)] for a, n in zip(starts, sizes)] if t is not None else None  # noqa: E731
        s["views"] = {n: cut(s[n]) for n in ("p", "m", "v", "p16", "p8")} | {n: cut(s[n], BLOCK) for n in ("me", "ve")}
    return s


def work(case):
    op = case["op"]
    if op == "table":
        n = case["N"] * (case["rot"] // 2)
        return {"bytes": 8 * n, "flops": 20 * n}
    if op in ("rope_fwd", "rope_bwd"):
        T, W, qk = case["T"], (case["Hq"] + 2 * case["Hkv"]) * case["d"], (case["Hq"] + case["Hkv"]) * case["d"]
        table = 4 * case["rot"] * min(T, case["N"]) + (8 * T if case["positions"] else 0)
        saved = 2 * T * qk if op == "rope_bwd" and case["mode"] != "none" else 0
        return {"bytes": T * W * (3 if case["codes"] else 4) + saved + table, "flops": 10 * T * W}
    if op == "norm_fwd":
        T, D = case["T"], case["D"]
        last = 1 if case["codes"] else 2 if case["pre"] else 0
        return {"bytes": T * D * (6 + 2 * (case["gate"] != "none") + last) + 4 * D * (case["pre"] + (case["post"] != "none"))
                + 4 * T * (case["pre"] + (case["post"] == "rms")), "flops": 12 * T * D}
    if op == "norm_bwd":
        T, D = case["T"], case["D"]
        gate, post, pre = case["gate"] != "none", case["post"] != "none", case["pre"]
        read = 4 * pre + 2 * case["dh"] + 2 * (post or gate) + 2 * gate
        return {"bytes": T * D * (read + 2 + (1 if case["codes"] else 2) + 2 * gate)
                + 4 * D * (pre + post) * (2 + case["accumulate"]) + 4 * T * (pre + (case["post"] == "rms")), "flops": 25 * T * D}
    n = sum(_sizes(case))
    states = 16 if case["bits"] == 32 else 4 + 4.0 / BLOCK
    return {"bytes": n * (8 + (4 if case["fp32"] else 2) + states + 2 + case["codes"]), "flops": 20 * n}


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"table": _table, "rope_fwd": _rope_fwd, "rope_bwd": _rope_bwd, "norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd,
            "adamw": _adamw}[s["op"]](s)


def _e4m3(v, scale):
    return (v.float() * scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _e5m2(v, scale):
    return (v.float() * scale).clamp(-E5M2_MAX, E5M2_MAX).to(torch.float8_e5m2)


def _amax(v):
    return v.float().abs().max().reshape(1)


def _table(s):
    if own:
        import paper_2505_20524_b200 as fp8
        kind = {"plain": fp8.ROPE_PLAIN, "linear": fp8.ROPE_LINEAR, "ntk": fp8.ROPE_NTK, "parts": fp8.ROPE_BY_PARTS}[s["scaling"]]
        fp8.fp8_rope_table(s["cos"], s["sin"], s["base"], kind, SCALING["factor"], SCALING["original_len"],
                           SCALING["turns_low"], SCALING["turns_high"], _magnitude(s["scaling"]))
        return {"cos": s["cos"], "sin": s["sin"]}
    turns = torch.arange(s["N"], device=DEVICE, dtype=torch.float64)[:, None] * _turns(s["rot"], s["scaling"], s["base"])
    angle = (turns - turns.round()) * (2.0 * math.pi)
    return {"cos": (angle.cos() * _magnitude(s["scaling"])).float(), "sin": (angle.sin() * _magnitude(s["scaling"])).float()}


def _mode(fp8, s):
    return {"rms": fp8.QK_RMS, "tanh": fp8.QK_TANH, "none": fp8.QK_NONE}[s["mode"]]


def _angles(s, T):
    """cos and sin of each token's position [T, 1, rot / 2], and whether the position is in the table [T, 1]."""
    pos = torch.arange(T, device=DEVICE) % s["N"] if s["pos"] is None else s["pos"].long()
    there = (pos >= 0) & (pos < s["N"])
    at = pos.clamp(0, s["N"] - 1)
    return s["cos"][at][:, None], s["sin"][at][:, None], there[:, None]


def _rotated(x, c, sn, rot, interleaved, sign):
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * c - sign * b * sn, b * c + sign * a * sn
    pair = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([pair, x[..., rot:]], -1)


def _rope_fwd(s):
    T, Hq, Hkv, d = s["T"], s["Hq"], s["Hkv"], s["d"]
    if own:
        import paper_2505_20524_b200 as fp8
        how = (_mode(fp8, s), ALPHA, s["eps"], s["cos"], s["sin"], s["pos"], s["interleaved"])
        if s["codes"]:
            fp8.fp8_rope_qkv_fwd_q(s["qkv"], Hq, Hkv, *how, s["scales"], fp8.E4M3, s["q"], s["k"], s["v"], amax_out=s["amax"])
            return {n: s[n].view(torch.float8_e4m3fn) for n in "qkv"} | {"amax": s["amax"]}
        fp8.fp8_rope_qkv_fwd(s["qkv"], Hq, Hkv, *how, s["q"], s["k"], s["v"], amax_out=s["amax"])
        return {n: s[n] for n in "qkv"} | {"amax": s["amax"]}
    x = s["qkv"].float().view(T, Hq + 2 * Hkv, d)
    qk, v = x[:, :Hq + Hkv], x[:, Hq + Hkv:]
    if s["mode"] == "rms":
        qk = qk * (1.0 / (qk.square().mean(-1, keepdim=True) + s["eps"]).sqrt())
    elif s["mode"] == "tanh":
        qk = torch.tanh(ALPHA * qk)
    c, sn, there = _angles(s, T)
    qk = _rotated(qk, c, sn, s["rot"], s["interleaved"], 1.0)
    out = torch.where(there[:, None], torch.cat([qk, v], 1), 0.0).bfloat16()
    parts = dict(zip("qkv", out.split([Hq, Hkv, Hkv], 1)))
    amax = torch.cat([_amax(parts[n]) for n in "qkv"])
    if s["codes"]:
        return {n: _e4m3(parts[n], s["scales"][i]) for i, n in enumerate("qkv")} | {"amax": amax}
    return {n: parts[n].contiguous() for n in "qkv"} | {"amax": amax}


def _rope_bwd(s):
    T, Hq, Hkv, d = s["T"], s["Hq"], s["Hkv"], s["d"]
    if own:
        import paper_2505_20524_b200 as fp8
        how = (s["qkv"], _mode(fp8, s), ALPHA, s["eps"], s["cos"], s["sin"], s["pos"], s["interleaved"])
        if s["codes"]:
            fp8.fp8_rope_qkv_bwd_q(s["dq"], s["dk"], s["dv"], *how, s["scale"], fp8.E5M2, s["dqkv"], amax_out=s["amax"])
            return {"dqkv": s["dqkv"].view(torch.float8_e5m2), "amax": s["amax"]}
        fp8.fp8_rope_qkv_bwd(s["dq"], s["dk"], s["dv"], *how, s["dqkv"], amax_out=s["amax"])
        return {"dqkv": s["dqkv"], "amax": s["amax"]}
    c, sn, there = _angles(s, T)
    u = _rotated(torch.cat([s["dq"], s["dk"]], 1).float(), c, sn, s["rot"], s["interleaved"], -1.0)
    if s["mode"] != "none":
        x = s["qkv"].float().view(T, Hq + 2 * Hkv, d)[:, :Hq + Hkv]
        if s["mode"] == "rms":
            r = 1.0 / (x.square().mean(-1, keepdim=True) + s["eps"]).sqrt()
            xh = x * r
            u = r * (u - xh * (u * xh).mean(-1, keepdim=True))
        else:
            u = ALPHA * (1.0 - torch.tanh(ALPHA * x).square()) * u
    out = torch.where(there[:, None], torch.cat([u, s["dv"].float()], 1), 0.0).bfloat16().view(T, -1)
    return {"dqkv": _e5m2(out, s["scale"]) if s["codes"] else out, "amax": _amax(out)}


def _norm_how(fp8, s):
    post = {"rms": fp8.NORM_RMS, "scale": fp8.NORM_LAYERSCALE, "none": fp8.NORM_NONE}[s["post"]]
    return post, fp8.GATE_SIGMOID if s["gate"] == "sigmoid" else fp8.GATE_LINEAR, s["a"], s["b"]


def _norm_fwd(s):
    if own:
        import paper_2505_20524_b200 as fp8
        ins = (s["x"], s["y"], s["gate_in"], s["gamma_post"], s["gamma_pre"], *_norm_how(fp8, s), s["eps"])
        if s["codes"]:
            fp8.fp8_block_norm_fwd_q(*ins, s["scale"], fp8.E4M3, s["h"], s["out"], s["out8"], r_post=s["r_post"], r_pre=s["r_pre"],
                                     amax_out=s["amax"])
            codes = {"codes": s["out8"].view(torch.float8_e4m3fn)}
        else:
            fp8.fp8_block_norm_fwd(*ins, s["h"], s["out"], r_post=s["r_post"], r_pre=s["r_pre"], amax_out=s["amax"])
            codes = {"out": s["out"]}
        return {"h": s["h"], "r_post": s["r_post"], "r_pre": s["r_pre"], "amax": s["amax"]} | codes
    z, r_post, r_pre = s["y"].float(), None, None
    if s["post"] == "rms":
        r_post = 1.0 / (z.square().mean(1) + s["eps"]).sqrt()
        z = z * r_post[:, None]
    if s["gamma_post"] is not None:
        z = z * s["gamma_post"]
    if s["gate_in"] is not None:
        gate = s["gate_in"].float()
        z = z * (1.0 / (1.0 + torch.exp(-gate)) if s["gate"] == "sigmoid" else gate)
    h = (s["a"] * s["x"].float() + s["b"] * z).bfloat16()
    out = h
    if s["pre"]:
        hf = h.float()
        r_pre = 1.0 / (hf.square().mean(1) + s["eps"]).sqrt()
        out = (hf * r_pre[:, None] * s["gamma_pre"]).bfloat16()
    got = {"h": h, "r_post": r_post, "r_pre": r_pre, "amax": _amax(out)}
    if s["codes"]:
        return got | {"codes": _e4m3(out, s["scale"])}
    return got | {"out": out if s["pre"] else None}


def _norm_bwd(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if "ws" not in s:
            s["ws"] = torch.empty(fp8.fp8_block_norm_bwd_workspace_bytes(s["T"], s["D"]), dtype=torch.uint8, device=DEVICE)
        ins = (s["dout"], s["dh"], s["h"], s["y"], s["gate_in"], s["gamma_post"], s["gamma_pre"], s["r_post"], s["r_pre"],
               *_norm_how(fp8, s))
        outs = (s["dgate"], s["dgamma_post"], s["dgamma_pre"], s["ws"])
        if s["codes"]:
            fp8.fp8_block_norm_bwd_q(*ins, s["scale"], fp8.E5M2, s["dx"], None, s["dy"], *outs, accumulate=s["accumulate"],
                                     amax_out=s["amax"])
        else:
            fp8.fp8_block_norm_bwd(*ins, s["dx"], s["dy"], *outs, accumulate=s["accumulate"], amax_out=s["amax"])
        dy = s["dy"].view(torch.float8_e5m2) if s["codes"] else s["dy"]
        return {"dx": s["dx"], "dy": dy, "dgate": s["dgate"], "dgamma_post": s["dgamma_post"], "dgamma_pre": s["dgamma_pre"],
                "amax": s["amax"]}
    total, dgamma_post, dgamma_pre, dgate = 0.0, None, None, None
    if s["pre"]:
        hh = s["h"].float() * s["r_pre"][:, None]
        dout = s["dout"].float()
        e = dout * s["gamma_pre"]
        total = s["r_pre"][:, None] * (e - hh * (e * hh).mean(1, keepdim=True))
        dgamma_pre = (dout * hh).sum(0)
    if s["dh"] is not None:
        total = total + s["dh"].float()
    dx = (s["a"] * total).bfloat16()
    dz = s["b"] * total
    yh = s["y"].float()
    if s["post"] == "rms":
        yh = yh * s["r_post"][:, None]
    if s["gate_in"] is not None:
        gate = s["gate_in"].float()
        z = yh * s["gamma_post"] if s["gamma_post"] is not None else yh
        if s["gate"] == "sigmoid":
            gate = 1.0 / (1.0 + torch.exp(-gate))
            dgate = (dz * z * gate * (1.0 - gate)).bfloat16()
        else:
            dgate = (dz * z).bfloat16()
        dz = dz * gate
    dy = dz
    if s["gamma_post"] is not None:
        dgamma_post = (dz * yh).sum(0)
        dy = dz * s["gamma_post"]
    if s["post"] == "rms":
        dy = s["r_post"][:, None] * (dy - yh * (dy * yh).mean(1, keepdim=True))
    dy = dy.bfloat16()
    if s["accumulate"]:
        if dgamma_post is not None:
            dgamma_post = s["dgamma_post"].add_(dgamma_post)
        if dgamma_pre is not None:
            dgamma_pre = s["dgamma_pre"].add_(dgamma_pre)
    return {"dx": dx, "dy": _e5m2(dy, s["scale"]) if s["codes"] else dy, "dgate": dgate, "dgamma_post": dgamma_post,
            "dgamma_pre": dgamma_pre, "amax": _amax(dy)}


def _adamw_out(s):
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    got = {"p": s["p"], "p16": s["p16"], "amax": s["amax"], "step": s["step"]}
    got |= {"m": s["m"].view(f8), "v": s["v"].view(f8), "me": s["me"].view(e8), "ve": s["ve"].view(e8)} if s["bits"] == 8 else \
        {"m": s["m"], "v": s["v"]}
    return got | ({"p8": s["p8"].view(f8)} if s["codes"] else {})


def _mix(x):
    """32-bit integers (held in 64) to 32-bit integers that look random: shifts and products, modulo 2^32."""
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(s, t):
    """32 bits for each element: a function of the seed, the step, the tensor's number and the element's index."""
    key = _mix(_mix(_mix(torch.full_like(t, s["seed"] & 0xFFFFFFFF)) ^ (s["seed"] >> 32)) ^ t)
    key = _mix((key + torch.arange(s["tensors"], device=DEVICE)) & 0xFFFFFFFF)
    key = _mix(key)                                           # (of the index's upper half, 0 for all of these tensors)
    index = torch.arange(s["p"].numel(), device=DEVICE) - s["starts"].repeat_interleave(s["counts"])
    return _mix((key.repeat_interleave(s["counts"]) + index) & 0xFFFFFFFF)


def _encode_random(x, bits, floor):
    """E4M3 codes of `x` under a power of two per block, rounded up with the probability of the part that is cut off: 16 random
    bits under the last bit that stays.  `floor`: values above zero get the smallest code at least."""
    x = x.view(-1, BLOCK)
    e = _block_exponent(x.abs().amax(1))
    y = x.abs() * _power(254 - e)[:, None]
    off = torch.where(y < 2.0 ** -6, 2.0 ** -6, 0.0)          # below the normal numbers the step stays 2^-9
    z = ((y + off).view(torch.int32) + (bits.view(-1, BLOCK) << 4).to(torch.int32) & -0x100000).view(torch.float32) - off
    if floor:
        z = torch.where((x > 0) & (z == 0), 2.0 ** -9, z)
    return torch.copysign(z, x).to(torch.float8_e4m3fn).view(torch.uint8).view(-1), e.to(torch.uint8)


def _adamw(s):
    if own:
        import paper_2505_20524_b200 as fp8
        if "items" not in s:
            v = s["views"]
            s["items"] = fp8.fp8_adamw_items(v["p"], s["grads"], v["m"], v["v"], s["decay"], m_exps=v["me"], v_exps=v["ve"],
                                             params16=v["p16"], params8=v["p8"], q_scales=s["q_scale"], amaxes=s["amax"], fmt=fp8.E4M3)
            s["ws"] = torch.empty(fp8.fp8_adamw_workspace_bytes(s["items"]), dtype=torch.uint8, device=DEVICE)
        fp8.fp8_adamw(s["items"], s["lr"], s["step"], s["beta1"], s["beta2"], s["adam_eps"], s["ws"], norm=s["norm"],
                      max_norm=s["max_norm"], seed=s["seed"])
        return _adamw_out(s)
    b1, b2 = s["beta1"], s["beta2"]
    s["step"] += 1
    t = s["step"].double()
    c1, c2 = (1.0 - b1 ** t).float(), (1.0 - b2 ** t).sqrt().float()
    factor = (s["max_norm"] / (s["norm"] + 1e-6)).clamp(max=1.0)
    g = torch.cat([x for pair in zip(s["grads"], s["gaps"]) for x in pair]).float() * factor
    if s["bits"] == 8:
        m = s["m"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * _power(s["me"])[:, None]
        r = s["v"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * _power(s["ve"])[:, None]
        m, v = m.view(-1), r.view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    r = v.sqrt()
    decay = (1.0 - s["lr"] * s["decays"]).repeat_interleave(s["counts"])
    s["p"].copy_(s["p"] * decay - (s["lr"] / c1) * (m / (r / c2 + s["adam_eps"])))
    s["p16"].copy_(s["p"])
    if s["bits"] == 8:
        bits = _random_bits(s, s["step"].long())
        s["m"], s["me"] = _encode_random(m, bits & 0xFFFF, False)
        s["v"], s["ve"] = _encode_random(r, bits >> 16, True)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    per_block = s["p16"].float().view(-1, BLOCK).abs().amax(1)
    block_of = torch.arange(s["tensors"], device=DEVICE).repeat_interleave(s["counts"] // BLOCK)
    s["amax"] = torch.zeros(s["tensors"], device=DEVICE).scatter_reduce_(0, block_of, per_block, "amax")
    if s["codes"]:
        s["p8"] = _e4m3(s["p16"], s["q_scale"].repeat_interleave(s["counts"])).view(torch.uint8)
    return _adamw_out(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def _codes_e5m2(x, scale):
    """What the gradient's codes stand for: the nearest of four values per power of two."""
    y = (x * scale.double()).clamp(-E5M2_MAX, E5M2_MAX)
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y).exponent.clamp(min=-13) - 3)
    return (y / step).round() * step


def exact(case, seed):
    f64, op = torch.float64, case["op"]
    s = prepare(case, seed)
    if op == "table":
        n = torch.arange(case["N"], device=DEVICE, dtype=f64)
        angle = torch.outer(n, _turns(case["rot"], case["scaling"], s["base"]) * 2.0 * math.pi)
        z = torch.polar(torch.full_like(angle, _magnitude(case["scaling"])), angle)
        return {"cos": z.real, "sin": z.imag}
    if op in ("rope_fwd", "rope_bwd"):
        T, Hq, Hkv, d, rot = case["T"], case["Hq"], case["Hkv"], case["d"], case["rot"]
        pos = s["pos"].long() if s["pos"] is not None else torch.arange(T, device=DEVICE) % case["N"]
        known = (pos >= 0) & (pos < case["N"])
        turn = torch.complex(s["cos"].double(), s["sin"].double())[torch.where(known, pos, 0)].unsqueeze(1)
        first = torch.arange(0, rot, 2) if case["interleaved"] else torch.arange(rot // 2)
        second = first + (1 if case["interleaved"] else rot // 2)
        qkv = s["qkv"].double().view(T, -1, d) * known.view(T, 1, 1)

        def block(x):
            if case["mode"] == "rms":
                x = x * (x.square().sum(-1, keepdim=True) / d + s["eps"]) ** -0.5
            elif case["mode"] == "tanh":
                x = (ALPHA * x).tanh()
            z = torch.complex(x[..., first], x[..., second]) * turn
            return x.index_copy(-1, first.to(DEVICE), z.real).index_copy(-1, second.to(DEVICE), z.imag)

        if op == "rope_fwd":
            y = torch.cat([block(qkv[:, :Hq + Hkv]), qkv[:, Hq + Hkv:]], 1) * known.view(T, 1, 1)
            parts = y.split([Hq, Hkv, Hkv], 1)
            if case["codes"]:
                parts = [(p * s["scales"][i].double()).clamp(-E4M3_MAX, E4M3_MAX) for i, p in enumerate(parts)]
            return {n: p for n, p in zip("qkv", parts)} | {"amax": None}
        with torch.enable_grad():
            x = qkv[:, :Hq + Hkv].clone().requires_grad_()
            grad, = torch.autograd.grad(block(x), x, torch.cat([s["dq"], s["dk"]], 1).double())
        grad = torch.cat([grad, s["dv"].double()], 1).view(T, -1)
        grad[~known] = 0.0
        if case["codes"]:
            grad = _codes_e5m2(grad, s["scale"])
        return {"dqkv": grad, "amax": None}
    if op in ("norm_fwd", "norm_bwd"):
        rms = lambda v: (v.square().sum(1) / case["D"] + s["eps"]) ** -0.5  # noqa: E731

        def share(y, gate, gamma):
            """The block's share of the residual stream, but for its scale."""
            if case["post"] == "rms":
                y = y * rms(y).unsqueeze(1)
            if gamma is not None:
                y = gamma * y
            return y if gate is None else torch.sigmoid(gate) * y if case["gate"] == "sigmoid" else gate * y

        wide = lambda n: None if s[n] is None else s[n].double()  # noqa: E731
        y, gate, gamma, gamma_pre = wide("y"), wide("gate_in"), wide("gamma_post"), wide("gamma_pre")
        if op == "norm_fwd":
            h = s["a"] * s["x"].double() + s["b"] * share(y, gate, gamma)
            stored = h.bfloat16().double()                    # the norm in front is that of the stored sum
            got = {"h": h, "r_post": rms(y) if case["post"] == "rms" else None, "r_pre": rms(stored) if case["pre"] else None,
                   "amax": None}
            out = gamma_pre * stored * rms(stored).unsqueeze(1) if case["pre"] else stored
            if case["codes"]:
                return got | {"codes": (out * s["scale"].double()).clamp(-E4M3_MAX, E4M3_MAX)}
            return got | {"out": out if case["pre"] else None}
        with torch.enable_grad():
            leaf = lambda v: None if v is None else v.requires_grad_()  # noqa: E731
            h, y, gate, gamma, gamma_pre = (leaf(v) for v in (s["h"].double(), y, gate, gamma, gamma_pre))
            total, dgamma_pre = torch.zeros_like(h), None
            if case["pre"]:
                total, dgamma_pre = torch.autograd.grad(h * rms(h).unsqueeze(1) * gamma_pre, (h, gamma_pre), s["dout"].double())
            if case["dh"]:
                total = total + s["dh"].double()
            ins = [v for v in (y, gate, gamma) if v is not None]
            grads = iter(torch.autograd.grad(share(y, gate, gamma) * 1.0, ins, s["b"] * total))
            dy = next(grads)
            dgate = next(grads) if gate is not None else None
            dgamma = next(grads) if gamma is not None else None
        if case["accumulate"]:
            dgamma = None if dgamma is None else dgamma + s["dgamma_post"].double()
            dgamma_pre = None if dgamma_pre is None else dgamma_pre + s["dgamma_pre"].double()
        if case["codes"]:
            dy = _codes_e5m2(dy, s["scale"])
        return {"dx": s["a"] * total, "dy": dy, "dgate": dgate, "dgamma_post": dgamma, "dgamma_pre": dgamma_pre, "amax": None}
    b1, b2, lr, t = s["beta1"], s["beta2"], float(s["lr"]), 101
    clip = min(1.0, s["max_norm"] / (float(s["norm"]) + 1e-6))
    flat = torch.zeros(s["p"].numel(), dtype=f64, device=DEVICE)
    decay = torch.zeros_like(flat)
    for start, grad, wd in zip(s["starts"].tolist(), s["grads"], s["decay"]):
        flat[start:start + grad.numel()] = grad.double() * clip
        decay[start:start + grad.numel()] = wd
    if case["bits"] == 8:
        value = lambda code, e: torch.ldexp(code.view(torch.float8_e4m3fn).double().view(-1, BLOCK), e.int()[:, None] - 127).view(-1)  # noqa: E731
        m, v = value(s["m"], s["me"]), value(s["v"], s["ve"]) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = m + (1.0 - b1) * (flat - m)
    v = v + (1.0 - b2) * (flat ** 2 - v)
    p = s["p"].double()
    p = p - lr * decay * p - lr * (m / (1.0 - b1 ** t)) / ((v / (1.0 - b2 ** t)) ** 0.5 + s["adam_eps"])
    got = {"p": p, "p16": p, "amax": None, "step": None}
    if case["codes"]:
        scale = torch.cat([q.double().expand(n) for q, n in zip(s["q_scale"], s["counts"].tolist())])
        got["p8"] = (p * scale).clamp(-E4M3_MAX, E4M3_MAX)
    if case["bits"] == 32:
        return got | {"m": m, "v": v}
    # what is stored in 8 bits, before its rounding: the values over their block's power of two
    for n, x in (("m", m), ("v", v ** 0.5)):
        rows = x.view(-1, BLOCK)
        e = torch.ceil(torch.log2(rows.abs().amax(1) / E4M3_MAX)).clamp(min=-126.0)
        e = torch.where(rows.abs().amax(1) > 0, e, torch.full_like(e, -126.0))
        got[n], got[n + "e"] = (rows * 2.0 ** -e[:, None]).view(-1), 2.0 ** e
    return got
