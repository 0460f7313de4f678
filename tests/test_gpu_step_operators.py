"""GPU parity of the operators around a step's FP8 products: token embedding and its gradient, layer norm forward and
backward, router with balance loss and gradient, gradient norm and clipping, against plain evaluations in 64 bits.

Tolerances.  u = 2^-24 is half a step of FP32, h = eps / 2 half a step of the output's type.  A sum of n FP32 terms in any
order is off by at most n u times the sum of their magnitudes (to first order); products and the function calls add a few u
per term.  Each test states its n.
"""
import math

import numpy as np
import pytest
import torch

import paper_2505_20524_b200 as fp8

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rnd(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def scalar(v):
    return torch.full((1,), float(v), device="cuda")


def ws_of(n):
    return torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda")       # scratch needs no preparation


def within(got, ref, tol):
    """|got - ref| <= tol elementwise (all in 64 bits); the message names the worst element."""
    d = (got.to(F64) - ref).abs() - tol
    assert not torch.isnan(d).any()
    worst = int(d.argmax())
    assert d.max() <= 0, (worst, got.reshape(-1)[worst].item(), ref.reshape(-1)[worst].item(), tol.reshape(-1)[worst].item())


def codes_of(x, scale, fmt):
    out8 = torch.empty(x.shape, dtype=torch.uint8, device="cuda")
    fp8.fp8_cast(x.reshape(-1), scale, fmt, out8.reshape(-1))        # flat: any length
    return out8


# ------------------------------------------------------------------------------------------------ embedding
def token_ids(g, T, V, dtype=torch.int64):
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=dtype)
    if T > 3:
        ids[T // 2] = -1
        ids[T // 3] = V
        ids[1] = -(1 << 31) if dtype == torch.int32 else (1 << 40)
    return ids


@pytest.mark.parametrize("T,V,D", [(1, 1, 8), (3, 7, 16), (33, 100, 72), (257, 1000, 256), (130, 513, 1600), (65, 300, 4104)])
@pytest.mark.parametrize("tdt,idt", [(BF16, torch.int64), (F32, torch.int32), (BF16, torch.int32), (F32, torch.int64)])
def test_embedding_forward_is_one_product_and_one_rounding(T, V, D, tdt, idt):
    g = gen(T + V + D)
    table, ids, scale = rnd(g, V, D, std=0.02, dtype=tdt), token_ids(g, T, V, idt), 50.3
    there = (ids >= 0) & (ids < V)
    want = table[torch.where(there, ids, 0).long()].float() * scale
    want = torch.where(there[:, None], want, 0.0).to(BF16)
    out, a = torch.full((T, D), 7.0, dtype=BF16, device="cuda"), scalar(-1)
    fp8.fp8_embedding_fwd(table, ids, scale, out, a)
    assert torch.equal(out, want) and a.item() == want.float().abs().max().item()
    for fmt in (fp8.E4M3, fp8.E5M2):
        qs = scalar(37.0)
        out8, o2, a2 = torch.empty((T, D), dtype=torch.uint8, device="cuda"), torch.empty_like(out), scalar(-1)
        fp8.fp8_embedding_fwd_q(table, ids, scale, qs, fmt, o2, out8, a2)
        assert torch.equal(o2, want) and a2.item() == a.item() and torch.equal(out8, codes_of(want, qs, fmt))
        out8.fill_(0xEE)
        fp8.fp8_embedding_fwd_q(table, ids, scale, qs, fmt, None, out8)            # codes only
        assert torch.equal(out8, codes_of(want, qs, fmt))


def test_embedding_forward_zero_rows_for_padding_whatever_the_scale():
    table = torch.ones((4, 16), device="cuda")
    out = torch.empty((3, 16), dtype=BF16, device="cuda")
    fp8.fp8_embedding_fwd(table, torch.tensor([-1, 2, 4], device="cuda"), math.inf, out)
    assert (out[0] == 0).all() and (out[2] == 0).all() and torch.isinf(out[1]).all()


EMB_BWD = [  # T, V, D, id pattern
    (1, 1, 8, "random"), (1, 5, 8, "random"), (2, 3, 24, "same"), (31, 50, 16, "random"), (32, 50, 16, "same"),
    (33, 50, 16, "same"), (64, 50, 16, "same"), (100, 7, 2056, "random"), (1000, 100000, 64, "random"),
    (5000, 40, 72, "random"), (5000, 1000, 264, "same"), (4096, 3000, 128, "sorted"), (4097, 3000, 128, "runs32"),
    (70000, 1100, 8, "zipf"), (9000, (1 << 20) + 5, 8, "zipf"), (600001, 2000, 8, "zipf"), (77, 9, 40, "padding"),
    (2048, 1024, 8, "random"), (2049, 1023, 8, "random"), (700, 300, 4104, "zipf"), (2000, (1 << 20) - 1, 8, "zipf"),
    (3000, (1 << 20) - 1, 8, "zipf"), (66000, (1 << 20) - 1, 8, "zipf"), (16384, 512, 16, "same"), (65536, 513, 8, "sorted"),
    (65537, 513, 8, "runs32"),
    (4736, 700, 16, "zipf"), (4737, 700, 16, "zipf"), (257, 30, 8, "same"), (2049, 9, 8, "runs32"),
    (3000, 40000, 1024, "zipf"), (100, 70000, 264, "random"), (2100, 2500, 1024, "random"),      # first rows cleared apart: part, all
]


def pattern(g, T, V, kind):
    if kind == "same":
        return torch.full((T,), V - 1, device="cuda")
    if kind == "padding":
        return torch.full((T,), -100, device="cuda")
    if kind == "sorted":
        return torch.arange(T, device="cuda") * V // T
    if kind == "runs32":                                       # runs that end exactly at a work item's end
        return torch.arange(T, device="cuda") // 32 % V
    if kind == "zipf":
        u = torch.rand(T, generator=g, device="cuda", dtype=F64)
        ids = (torch.exp(u * math.log(V + 1.0)) - 1).long().clamp(0, V - 1)
        ids[torch.rand(T, generator=g, device="cuda") < 0.05] = -1
        return ids
    return token_ids(g, T, V)


@pytest.mark.parametrize("T,V,D,kind", EMB_BWD)
@pytest.mark.parametrize("dt,accumulate", [(BF16, False), (F32, False), (BF16, True), (F32, True)])
def test_embedding_gradient(T, V, D, kind, dt, accumulate):
    g = gen(T + 3 * V + D)
    ids, dy, scale = pattern(g, T, V, kind), rnd(g, T, D, dtype=BF16), 1.7
    ids = ids.to(torch.int32) if T % 2 else ids
    keep = (ids >= 0) & (ids < V)
    at, rows = ids[keep].long(), dy[keep].to(F64)
    total = torch.zeros((V, D), dtype=F64, device="cuda").index_add_(0, at, rows) * float(np.float32(scale))
    size = torch.zeros((V, D), dtype=F64, device="cuda").index_add_(0, at, rows.abs()) * float(np.float32(scale))
    n = torch.zeros(V, dtype=F64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=F64))
    got = rnd(g, V, D, dtype=dt) if accumulate else torch.full((V, D), math.nan, dtype=dt, device="cuda")
    old = got.clone()
    if accumulate:
        got[n == 0] = math.nan                                  # rows without a token are not read
        old[n == 0] = 0
        total += old.to(F64)
        size += old.to(F64).abs()
    first = got.clone()
    ws = ws_of(fp8.fp8_embedding_bwd_workspace_bytes(T, V, D))
    fp8.fp8_embedding_bwd(dy, ids, scale, got, ws, accumulate=accumulate)
    if accumulate:
        assert torch.isnan(got[n == 0]).all()
        got[n == 0] = 0
    # n additions, the product with scale (and the addition of the old value) in one step
    within(got, total, HALF[dt] * total.abs() + (n + 2)[:, None] * U * size * (1 + 2 ** -7))
    # the same call again gives the same bits
    fp8.fp8_embedding_bwd(dy, ids, scale, first, ws, accumulate=accumulate)
    if accumulate:
        first[n == 0] = 0
    assert torch.equal(first, got)


def test_embedding_gradient_ignores_what_stands_at_padded_positions():
    T, V, D = 3000, 50, 64
    g = gen(6)
    ids, dy = torch.randint(0, V, (T,), generator=g, device="cuda"), rnd(g, T, D, dtype=BF16)
    pad = torch.rand(T, generator=g, device="cuda") < 0.3
    ids[pad] = -1
    clean, dirty = torch.empty((V, D), device="cuda"), torch.empty((V, D), device="cuda")
    ws = ws_of(fp8.fp8_embedding_bwd_workspace_bytes(T, V, D))
    fp8.fp8_embedding_bwd(dy, ids, 1.0, clean, ws)
    dy[pad] = math.nan
    fp8.fp8_embedding_bwd(dy, ids, 1.0, dirty, ws)
    assert torch.equal(clean, dirty) and torch.isfinite(dirty).all()


def test_embedding_takes_slices_of_the_ids():
    """ids need no more than their own alignment: the tokens shifted by one."""
    T, V, D = 33, 60, 32
    g = gen(7)
    table, dy = rnd(g, V, D), rnd(g, T, D, dtype=BF16)
    for dt in (torch.int64, torch.int32):
        ids = torch.randint(0, V, (T + 1,), generator=g, device="cuda", dtype=dt)
        out = torch.empty((T, D), dtype=BF16, device="cuda")
        fp8.fp8_embedding_fwd(table, ids[1:], 1.0, out)
        assert torch.equal(out, table[ids[1:].long()].to(BF16))
        a, b = torch.empty((V, D), device="cuda"), torch.empty((V, D), device="cuda")
        ws = ws_of(fp8.fp8_embedding_bwd_workspace_bytes(T, V, D))
        fp8.fp8_embedding_bwd(dy, ids[1:], 1.0, a, ws)
        fp8.fp8_embedding_bwd(dy, ids[1:].clone(), 1.0, b, ws)
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ layer norm
LN = [(1, 8), (5, 64), (9, 256), (17, 264), (33, 512), (7, 520), (65, 1024), (33, 1032), (3, 2048), (130, 2056), (70, 4096),
      (11, 4104), (19, 8192), (6, 8200), (5, 16384), (1, 16376), (1200, 128), (700, 1536),
      # several rows to a warp: the last ones missing, lanes without columns, more than one turn of all warps
      (1, 24), (6, 8), (700, 8), (63, 40), (130, 72), (33, 200), (1300, 248), (9001, 136), (250001, 8)]


def ln_data(T, D, seed=0, offset=0.5):
    g = gen(T * 31 + D + seed)
    x = rnd(g, T, D) * torch.where(torch.rand(D, generator=g, device="cuda") < 0.02, 20.0, 1.0) + offset
    return g, x.to(BF16), 1 + 0.2 * rnd(g, D), 0.3 * rnd(g, D)


def ln_reference(x, gamma, beta, eps, res=None):
    xd = x.to(F64)
    mu = xd.mean(1, keepdim=True)
    rs = ((xd - mu).square().mean(1, keepdim=True) + eps).rsqrt()
    y = (xd - mu) * rs * gamma.to(F64) + beta.to(F64)
    size = gamma.to(F64).abs() * rs * (xd.abs() + xd.abs().mean(1, keepdim=True)) + beta.to(F64).abs()
    if res is not None:
        y, size = y + res.to(F64), size + res.to(F64).abs()
    return y, mu[:, 0], rs[:, 0], size


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,D", LN)
def test_layernorm_forward(T, D, residual):
    g, x, gamma, beta = ln_data(T, D)
    eps = 1e-5
    res = rnd(g, T, D, dtype=BF16) if residual else None
    want, mu, rs, size = ln_reference(x, gamma, beta, float(np.float32(eps)), res)
    out, mean, rstd, a = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), scalar(-1)
    fp8.fp8_layernorm_fwd(x, gamma, beta, eps, out, mean=mean, rstd=rstd, residual=res, amax_out=a)
    # row sums: 16 terms per thread, 5 shuffle steps, up to 32 warps: n = 64 covers them, and the same again for the squares;
    # half of that reaches rstd
    within(mean, mu, 66 * U * x.to(F64).abs().mean(1))
    within(rstd, rs, 160 * U * rs)
    within(out, want, HALF[BF16] * want.abs() + 240 * U * size * (1 + 2 ** -7))
    assert a.item() == out.float().abs().max().item()
    for fmt in (fp8.E4M3, fp8.E5M2):
        qs, o2, out8, a2 = scalar(11.0), torch.empty_like(x), torch.empty(x.shape, dtype=torch.uint8, device="cuda"), scalar(-1)
        fp8.fp8_layernorm_fwd_q(x, gamma, beta, eps, qs, fmt, o2, out8, residual=res, amax_out=a2)
        assert torch.equal(o2, out) and a2.item() == a.item() and torch.equal(out8, codes_of(out, qs, fmt))
    # in place: over x, and over the residual
    xc = x.clone()
    fp8.fp8_layernorm_fwd(xc, gamma, beta, eps, xc, residual=res)
    assert torch.equal(xc, out)
    if residual:
        rc = res.clone()
        fp8.fp8_layernorm_fwd(x, gamma, beta, eps, rc, residual=rc)
        assert torch.equal(rc, out)


def test_layernorm_forward_keeps_its_digits_far_from_zero():
    """Rows whose mean is 500 times their deviation: the squares are taken of the distances from the mean."""
    T, D = 9, 4096
    g = gen(3)
    x = (1000.0 + 2.0 * torch.randint(-4, 5, (T, D), generator=g, device="cuda")).to(BF16)      # exact in BF16 (steps of 4 round)
    gamma, beta = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    _, mu, rs, _ = ln_reference(x, gamma, beta, 0.0)
    out, mean, rstd = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    fp8.fp8_layernorm_fwd(x, gamma, beta, 0.0, out, mean=mean, rstd=rstd)
    within(mean, mu, 66 * U * mu.abs())
    # the mean's error e enters the variance as e^2: (66 u 1000)^2 is far below u of the variance; the sum of squares as before
    within(rstd, rs, 160 * U * rs + rs ** 3 * (66 * U * 1000) ** 2)


def test_amax_of_large_outputs():
    """From 2^24 elements on the amax is set to zero by a kernel beside the main one: the same results, stale values ignored,
    call after call on the same scalar."""
    T, D, V = 4100, 4096, 300
    g, x, gamma, beta = ln_data(T, D, seed=5)
    table, ids = rnd(g, V, D, std=0.02, dtype=BF16), token_ids(g, T, V)
    out, a = torch.empty_like(x), scalar(1e30)
    for k in range(3):
        fp8.fp8_layernorm_fwd(x, gamma, beta, 1e-5, out, amax_out=a)
        assert a.item() == out.float().abs().max().item()
        fp8.fp8_embedding_fwd(table, ids, 50.0 / (k + 1), out, a)
        assert a.item() == out.float().abs().max().item()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fp8.fp8_layernorm_fwd(x, gamma, beta, 1e-5, out, amax_out=a)
    x.mul_(0.5)
    for _ in range(2):
        a.fill_(1e30)
        graph.replay()
        assert a.item() == out.float().abs().max().item()


@pytest.mark.parametrize("T,D", [(1, 8), (1, 16384), (8, 4096), (9, 4096), (16, 2048), (17, 2048), (8, 16384), (9, 16384), (129, 256),
                                 (257, 256), (300, 8)])
def test_amax_of_few_blocks(T, D):
    """Grids that are one cluster, and those just above: eagerly, on two streams, replayed; stale values ignored, zero for zeros."""
    g, x, gamma, beta = ln_data(T, D, seed=6)
    table, ids = rnd(g, 50, D, std=0.02), token_ids(g, T, 50)
    outs, amax = [torch.empty_like(x) for _ in range(2)], [scalar(1e30), scalar(1e30)]
    run = [lambda: fp8.fp8_layernorm_fwd(x, gamma, beta, 1e-5, outs[0], amax_out=amax[0]),
           lambda: fp8.fp8_embedding_fwd(table, ids, 50.0, outs[1], amax[1])]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for f, s in zip(run, side):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                f()
        torch.cuda.synchronize()
        for o, a in zip(outs, amax):
            assert a.item() == o.float().abs().max().item()
            a.fill_(1e30)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for f in run:
            f()
    for scale in (0.25, 0.0):
        x.mul_(scale)
        table.mul_(scale)
        if scale == 0.0:
            beta.zero_()
        for a in amax:
            a.fill_(1e30)
        graph.replay()
        for o, a in zip(outs, amax):
            assert a.item() == o.float().abs().max().item()
    assert amax[0].item() == 0.0 and amax[1].item() == 0.0


def test_layernorm_constant_rows_and_infinities():
    T, D = 3, 128
    x = torch.full((T, D), 2.5, dtype=BF16, device="cuda")
    x[1, 5] = math.inf
    x[2, 7] = math.nan
    gamma, beta = torch.ones(D, device="cuda"), torch.full((D,), 0.25, device="cuda")
    out, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
    fp8.fp8_layernorm_fwd(x, gamma, beta, 1e-6, out, rstd=rstd)
    assert (out[0] == 0.25).all() and abs(rstd[0].item() - 1000.0) <= 1000 * 4 * U + 1000 * 2 ** -22
    assert torch.isnan(out[1:]).all()


def ln_backward_reference(dout, x, gamma, mean, rstd):
    d, g = dout.to(F64), gamma.to(F64)
    xh = (x.to(F64) - mean.to(F64)[:, None]) * rstd.to(F64)[:, None]
    gd, r = d * g, rstd.to(F64)[:, None]
    dx = r * (gd - gd.mean(1, keepdim=True) - xh * (gd * xh).mean(1, keepdim=True))
    size = r * (gd.abs() + gd.abs().mean(1, keepdim=True) + xh.abs() * (gd * xh).abs().mean(1, keepdim=True))
    # xh itself: the difference is off by half a step of itself, the product again
    return dx, size, (d * xh).sum(0), (d * xh).abs().sum(0), d.sum(0), d.abs().sum(0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,D", LN + [(4099, 1032), (3000, 64), (2500, 2048)])
def test_layernorm_backward(T, D, accumulate):
    g, x, gamma, beta = ln_data(T, D, seed=1)
    dout = rnd(g, T, D, std=1e-2, dtype=BF16)
    _, mu, rs, _ = ln_reference(x, gamma, beta, 1e-5)
    mean, rstd = mu.float(), rs.float()
    want, size, wg, sg, wb, sb = ln_backward_reference(dout, x, gamma, mean, rstd)
    dx = torch.empty_like(x)
    dg, db = (rnd(g, D), rnd(g, D)) if accumulate else (torch.full((D,), math.nan, device="cuda") for _ in range(2))
    dg0, db0 = dg.clone(), db.clone()
    if accumulate:
        wg, wb, sg, sb = wg + dg0.to(F64), wb + db0.to(F64), sg + dg0.to(F64).abs(), sb + db0.to(F64).abs()
    ws = ws_of(fp8.fp8_layernorm_bwd_workspace_bytes(T, D))
    fp8.fp8_layernorm_bwd(dout, x, gamma, mean, rstd, dx, dg, db, ws, accumulate=accumulate)
    # row sums as in the forward (n = 64), about ten more operations on the way
    within(dx, want, HALF[BF16] * want.abs() + 96 * U * size * (1 + 2 ** -7))
    # over rows: at most ceil(T / 148) of them in one thread (every SM has a CTA once there are rows for it), then 8 warps and
    # 148 CTAs or fewer sums per thread
    n = -(-T // 148) + 256
    within(dg, wg, (n + 4) * U * sg)
    within(db, wb, n * U * sb)
    again = [torch.empty_like(dx), dg0.clone(), db0.clone()]
    fp8.fp8_layernorm_bwd(dout, x, gamma, mean, rstd, *again, ws, accumulate=accumulate)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dg) and torch.equal(again[2], db)
    for alias in ("dout", "x"):                                  # dx over one of its inputs
        dc, xc = dout.clone(), x.clone()
        o = dc if alias == "dout" else xc
        fp8.fp8_layernorm_bwd(dc, xc, gamma, mean, rstd, o, torch.empty_like(dg), torch.empty_like(db), ws)
        assert torch.equal(o, dx)


@pytest.mark.parametrize("D", [8, 24, 72, 200, 264, 520, 1032, 4104, 8200])
def test_layernorm_backward_where_mean_times_rstd_overflows(D):
    """A constant row far out: x - mean is zero, and nothing of the columns that a row does not have may come in."""
    g, x, gamma, _ = ln_data(5, D, seed=2)
    x[1], x[4] = 2.0 ** 120, -2.0 ** 126
    dout = rnd(g, 5, D, std=1e-2, dtype=BF16)
    _, mu, rs, _ = ln_reference(x, gamma, gamma, 1e-5)
    mean, rstd = mu.float(), rs.float()
    assert mean[1] == 2.0 ** 120 and torch.isinf(mean[1] * rstd[1])
    want, size, wg, sg, wb, sb = ln_backward_reference(dout, x, gamma, mean, rstd)
    dx, dg, db = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    fp8.fp8_layernorm_bwd(dout, x, gamma, mean, rstd, dx, dg, db, ws_of(fp8.fp8_layernorm_bwd_workspace_bytes(5, D)))
    # as in test_layernorm_backward: row sums of n = 64 terms, five rows
    within(dx, want, HALF[BF16] * want.abs() + 96 * U * size * (1 + 2 ** -7))
    within(dg, wg, 261 * U * sg)
    within(db, wb, 257 * U * sb)


def test_layernorm_gradient_against_differences():
    """Directional derivatives of sum(c * out) by central differences of the 64-bit forward, against the kernel's gradients."""
    T, D = 6, 96
    g, x, gamma, beta = ln_data(T, D, seed=2)
    c = rnd(g, T, D, dtype=BF16)
    _, mu, rs, _ = ln_reference(x, gamma, beta, 1e-5)
    dx, dg, db = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    fp8.fp8_layernorm_bwd(c, x, gamma, mu.float(), rs.float(), dx, dg, db, ws_of(fp8.fp8_layernorm_bwd_workspace_bytes(T, D)))

    def f(xd, gd, bd):
        m = xd.mean(1, keepdim=True)
        return (c.to(F64) * ((xd - m) * ((xd - m).square().mean(1, keepdim=True) + 1e-5).rsqrt() * gd + bd)).sum()

    for seed in range(3):
        h = gen(50 + seed)
        vx, vg, vb = rnd(h, T, D).to(F64), rnd(h, D).to(F64), rnd(h, D).to(F64)
        s = 1e-5
        args = (x.to(F64), gamma.to(F64), beta.to(F64))
        num = (f(*(a + s * v for a, v in zip(args, (vx, vg, vb)))) - f(*(a - s * v for a, v in zip(args, (vx, vg, vb))))) / (2 * s)
        parts = [(dx.to(F64) * vx), (dg.to(F64) * vg), (db.to(F64) * vb)]
        got = sum(p.sum() for p in parts)
        # dx is rounded to BF16 (half a step per term); the differences are good to about s^2 = 1e-10 of the size
        tol = HALF[BF16] * parts[0].abs().sum() + 1e-5 * sum(p.abs().sum() for p in parts)
        assert abs(num - got) <= tol


# ------------------------------------------------------------------------------------------------ router
def route_reference(logits, bias, k, normalize, cb, cz):
    l32 = logits.float()
    T, E = l32.shape
    broken = (torch.isnan(l32) | (l32 == math.inf)).any(1)
    routed = ~broken & (l32 > -math.inf).any(1)
    score = l32 if bias is None else l32 + bias
    score = torch.where(routed[:, None], score, -math.inf)
    v, i = torch.sort(score, dim=1, descending=True, stable=True)
    ok = v[:, :k] > -math.inf
    expert = torch.where(ok, i[:, :k], -1).int()
    l = l32.to(F64)
    p = torch.where(routed[:, None], torch.softmax(torch.where(routed[:, None], l, 0.0), 1), 0.0)
    idx = expert.clamp(min=0).long()
    if normalize:
        w = torch.softmax(torch.where(ok, l.gather(1, idx), -1e300), 1) * ok
    else:
        w = p.gather(1, idx) * ok
    w = torch.where(broken[:, None], math.nan, w)
    flat = expert.reshape(-1)
    counts = torch.stack([(flat == e).sum() for e in range(E)]).int()
    offsets = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), counts.cumsum(0).int()])
    order = torch.sort(torch.where(flat < 0, E, flat), stable=True)
    rows = torch.where(order.values < E, order.indices, -1).int()
    n = int((routed | broken).sum())
    lse = torch.where(routed, torch.logsumexp(torch.where(routed[:, None], l, 0.0), 1), 0.0)
    loss = torch.zeros(2, dtype=F64, device="cuda")
    if n:
        loss = torch.stack([cb * E * (counts.to(F64) / (k * n) * p.sum(0) / n).sum(), cz * lse.square().sum() / n])
    if broken.any():
        loss = torch.full_like(loss, math.nan)
    return dict(expert=expert, weight=w, counts=counts, offsets=offsets, rows=rows, n=n, loss=loss, p=p, lse=lse, routed=routed,
                broken=broken, ok=ok)


def route_outputs(T, E, k):
    i = dict(dtype=torch.int32, device="cuda")
    return dict(expert=torch.full((T, k), -7, **i), weight=torch.full((T, k), math.nan, device="cuda"), counts=torch.full((E,), -7, **i),
                offsets=torch.full((E + 1,), -7, **i), rows=torch.full((T * k,), -7, **i), n_routed=torch.full((1,), -7, **i),
                loss=torch.full((2,), -7.0, device="cuda"))


def route(logits, bias, k, normalize, cb, cz, rows=True):
    T, E = logits.shape
    o = route_outputs(T, E, k)
    fp8.fp8_moe_route(logits, bias, normalize, cb, cz, o["expert"], o["weight"], o["counts"], o["offsets"],
                      o["rows"] if rows else None, o["n_routed"], o["loss"], ws_of(fp8.fp8_moe_route_workspace_bytes(T, E)))
    return o


ROUTE = [(1, 1, 1), (1, 2, 2), (5, 7, 3), (33, 8, 2), (4097, 8, 2), (100, 9, 9), (50, 16, 16), (129, 17, 4), (64, 32, 8), (65, 33, 5),
         (300, 64, 6), (1000, 65, 1), (777, 128, 16), (40, 129, 8), (5001, 160, 6), (256, 256, 8), (2, 256, 16), (20000, 64, 2),
         # one kernel for few tokens, and the first size with two
         (1, 256, 16), (31, 200, 7), (224, 40, 4), (224, 256, 16), (225, 40, 4), (223, 128, 5),
         # both sides of the sizes from which a lane takes a token
         (4096, 8, 3), (8193, 1, 1), (9001, 8, 8), (8200, 5, 2), (12288, 16, 4), (12289, 16, 16), (12300, 11, 3), (32769, 16, 4),
         (33001, 9, 2)]
CB, CZ = float(np.float32(0.01)), float(np.float32(0.003))


@pytest.mark.parametrize("T,E,k", ROUTE)
@pytest.mark.parametrize("dt,normalize,with_bias", [(F32, True, True), (F32, False, False), (BF16, False, True), (BF16, True, False)])
def test_router_forward_and_gradient(T, E, k, dt, normalize, with_bias):
    g = gen(T * 7 + E + k)
    logits = rnd(g, T, E, std=2.0, dtype=dt)
    bias = 0.3 * rnd(g, E) if with_bias else None
    if T > 8 and E > 1:
        logits[torch.rand((T, E), generator=g, device="cuda") < 0.15] = -math.inf
        logits[3] = -math.inf                                    # a padded token
        logits[4] = 1.0                                          # all equal: the lowest experts
        logits[5] = -0.0
        logits[5, -1] = 0.0
        logits[6] = -math.inf
        logits[6, E // 2] = -3.0                                 # one expert left for k slots
        logits[7] = -30.0
        logits[7, 0] = torch.finfo(dt).min                       # the type's lowest value is a number
    r = route_reference(logits, bias, k, normalize, CB, CZ)
    o = route(logits, bias, k, normalize, CB, CZ)
    for name in ("expert", "counts", "offsets", "rows"):
        assert torch.equal(o[name], r[name]), name
    assert o["n_routed"].item() == r["n"]
    finite = torch.where(logits.float().abs() > 200, 0.0, logits.float()).abs().max().item()
    # exp of an FP32 difference: half a step of the difference (at most 2 * finite), expf itself 2 steps; sum of E; a product.
    # Logits beyond 200 in size are masks here: their probability is 0 on both sides
    rel = (4 * finite + E / 8 + 24) * U
    within(o["weight"], r["weight"], rel * r["weight"] + 1e-37)
    n = max(1, r["n"])
    chain = -(-T // 148) + 64                                    # tokens that one lane adds up, then 8 warps
    within(o["loss"], r["loss"], (rel + chain * U) * r["loss"] + torch.stack([torch.zeros((), dtype=F64, device="cuda"),
           CZ * 2 * r["lse"].abs().sum() / n * (E / 8 + 8 + 2 * finite) * U]))
    o2 = route(logits, bias, k, normalize, CB, CZ, rows=False)
    for name in o:
        assert torch.equal(o2[name], o[name]) or name == "rows", name
    assert (o2["rows"] == -7).all()
    # gradient
    dweight, dloss = rnd(g, T, k), scalar(1.5)
    dl = torch.full((T, E), math.nan, dtype=dt, device="cuda")
    fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], normalize, CB, CZ, dloss, dweight, dl)
    idx, ok = r["expert"].clamp(min=0).long(), r["ok"]
    dw = torch.where(ok, dweight.to(F64), 0.0)
    u = (1.5 * CB * E * r["counts"].to(F64) / (k * n * n)).expand(T, E).clone()
    if not normalize:
        u.scatter_add_(1, idx, dw)
    p = r["p"]
    zterm = 1.5 * CZ * 2 / n * r["lse"][:, None] * p
    want = p * (u - (u * p).sum(1, keepdim=True)) + zterm
    size = p * (u.abs() + (u.abs() * p).sum(1, keepdim=True)) + zterm.abs()
    if normalize:
        w = r["weight"]
        want.scatter_add_(1, idx, w * (dw - (dw * w).sum(1, keepdim=True)))
        size.scatter_add_(1, idx, w * (dw.abs() + (dw.abs() * w).sum(1, keepdim=True)))
    within(dl, want, HALF[dt] * want.abs() + (4 * rel + (E + 32) * U) * size + 1e-37)
    # without the optional inputs: the losses' gradient alone
    dl2 = torch.full((T, E), math.nan, dtype=dt, device="cuda")
    fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], normalize, CB, CZ, None, None, dl2)
    u = (CB * E * r["counts"].to(F64) / (k * n * n)).expand(T, E)
    want = p * (u - (u * p).sum(1, keepdim=True)) + zterm / 1.5
    size = p * (u + (u * p).sum(1, keepdim=True)) + zterm.abs()
    within(dl2, want, HALF[dt] * want.abs() + (4 * rel + (E + 32) * U) * size + 1e-37)


def test_router_gradient_against_differences():
    T, E, k = 9, 12, 3
    g = gen(4)
    logits, dweight = rnd(g, T, E), rnd(g, T, k)
    for normalize in (False, True):
        o = route(logits, None, k, normalize, CB, CZ)
        dl = torch.empty_like(logits)
        fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], normalize, CB, CZ, None, dweight, dl)
        idx = o["expert"].long()

        def f(l):                                                # the choice and the counts held fixed
            p = torch.softmax(l, 1)
            w = torch.softmax(l.gather(1, idx), 1) if normalize else p.gather(1, idx)
            return (CB * E * (o["counts"].to(F64) / (k * T) * p.mean(0)).sum() + CZ * torch.logsumexp(l, 1).square().mean()
                    + (w * dweight.to(F64)).sum())

        for seed in range(3):
            v, s = rnd(gen(90 + seed), T, E).to(F64), 1e-5
            num = (f(logits.to(F64) + s * v) - f(logits.to(F64) - s * v)) / (2 * s)
            got = (dl.to(F64) * v).sum()
            assert abs(num - got) <= 1e-5 * (dl.to(F64) * v).abs().sum()


def test_router_nothing_routed_and_broken_rows():
    T, E, k = 40, 10, 3
    o = route(torch.full((T, E), -math.inf, device="cuda"), None, k, True, CB, CZ)
    assert (o["expert"] == -1).all() and (o["weight"] == 0).all() and (o["counts"] == 0).all() and (o["offsets"] == 0).all()
    assert (o["rows"] == -1).all() and o["n_routed"].item() == 0 and (o["loss"] == 0).all()
    dl = torch.full((T, E), math.nan, device="cuda")
    fp8.fp8_moe_route_bwd(torch.full((T, E), -math.inf, device="cuda"), o["expert"], o["counts"], o["n_routed"], True, CB, CZ, None,
                          torch.ones((T, k), device="cuda"), dl)
    assert (dl == 0).all()
    for bad in (math.nan, math.inf):
        logits = rnd(gen(8), T, E)
        logits[7, 2] = bad
        r = route_reference(logits, None, k, False, CB, CZ)
        o = route(logits, None, k, False, CB, CZ)
        for name in ("expert", "counts", "offsets", "rows"):
            assert torch.equal(o[name], r[name]), name
        assert torch.isnan(o["weight"][7]).all() and torch.isnan(o["loss"]).all() and not torch.isnan(o["weight"][:7]).any()
        dl = torch.empty_like(logits)
        fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], False, CB, CZ, None, None, dl)
        assert torch.isnan(dl[7]).all() and not torch.isnan(dl[:7]).any() and not torch.isnan(dl[8:]).any()


@pytest.mark.parametrize("dt", [F32, BF16])
def test_router_rows_of_the_types_lowest_value(dt):
    """Equal numbers like any other: the lowest experts, equal weights; lse^2 lies beyond FP32, which a zero z_coef ignores."""
    T, E, k = 5, 8, 2
    logits = rnd(gen(10), T, E, dtype=dt)
    logits[2] = torch.finfo(dt).min
    o = route(logits, None, k, False, CB, 0.0)
    assert o["expert"][2].tolist() == [0, 1] and (o["weight"][2] == 0.125).all() and o["n_routed"].item() == T
    assert o["loss"][1] == 0 and torch.isfinite(o["loss"][0])
    assert torch.isinf(route(logits, None, k, False, CB, CZ)["loss"][1])
    dl = torch.empty_like(logits)
    fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], False, CB, 0.0, None, torch.ones((T, k), device="cuda"), dl)
    assert torch.isfinite(dl).all()


def test_router_bias_of_minus_infinity_closes_an_expert():
    logits = rnd(gen(9), 50, 6)
    bias = torch.zeros(6, device="cuda")
    bias[2] = -math.inf
    o = route(logits, bias, 6, True, CB, CZ)
    assert (o["expert"][:, 5] == -1).all() and o["counts"][2] == 0 and (o["expert"] != 2).all()
    assert torch.equal(o["weight"][:, 5], torch.zeros(50, device="cuda"))


def test_router_feeds_the_grouped_products():
    """Offsets and rows as the grouped FP8 product reads them: every token's copies meet their expert's weight."""
    T, E, k, K, N = 70, 5, 2, 64, 32
    g = gen(21)
    x, w = rnd(g, T, K, dtype=BF16), rnd(g, E, N, K, dtype=BF16)
    logits = rnd(g, T, E)
    logits[11] = -math.inf
    o = route(logits, None, k, True, CB, CZ)
    used = int(o["offsets"][E].item())
    x8, w8 = torch.empty((T, K), dtype=torch.uint8, device="cuda"), torch.empty((E, N, K), dtype=torch.uint8, device="cuda")
    a, sx, sxi, sw, swi = (scalar(0) for _ in range(5))
    fp8.fp8_quantize(x, fp8.E4M3, x8, None, a, sx, sxi)
    fp8.fp8_quantize(w, fp8.E4M3, w8, None, a, sw, swi)
    sorted8 = torch.zeros((T * k, K), dtype=torch.uint8, device="cuda")
    sorted8[:used] = x8[(o["rows"][:used] // k).long()]
    y = torch.zeros((T * k, N), dtype=F32, device="cuda")
    fp8.fp8_grouped_linear_fwd(sorted8, w8, sxi, swi.expand(E).contiguous(), o["offsets"], y)
    got = torch.zeros((T, N), dtype=F64, device="cuda")
    flat = o["rows"][:used].long()
    got.index_add_(0, flat // k, y[:used].to(F64) * o["weight"].reshape(-1)[flat].to(F64)[:, None])
    xd, wd = x8.view(torch.float8_e4m3fn).to(F64) * sxi.item(), w8.view(torch.float8_e4m3fn).to(F64) * swi.item()
    want, size = torch.zeros((T, N), dtype=F64, device="cuda"), torch.zeros((T, N), dtype=F64, device="cuda")
    for j in range(k):
        e = o["expert"][:, j].long()
        we = o["weight"][:, j].to(F64)[:, None] * (e >= 0)[:, None]
        want += we * torch.einsum("tk,tnk->tn", xd, wd[e.clamp(min=0)])
        size += we * torch.einsum("tk,tnk->tn", xd.abs(), wd[e.clamp(min=0)].abs())
    # FP32 accumulation of 64 products on the tensor cores (2^-22 of the sum of magnitudes, as the products' tests state) and
    # the descale's two products
    within(got, want, (2.0 ** -19) * size)


# ------------------------------------------------------------------------------------------------ gradient norm and clip
def grad_sets(kind):
    g = gen(77)
    if kind == "one":
        return [rnd(g, 1)]
    if kind == "mixed":
        return [rnd(g, n, dtype=(BF16 if i % 2 else F32), std=0.1 * (1 + i % 3)) for i, n in enumerate(
            [1, 7, 8, 9, 8191, 8192, 8193, 65537, 3, 0, 100000, 15, 256 * 8192 + 5])]
    if kind == "many":                                           # more tensors than one launch takes
        return [rnd(g, 1 + (i * 37) % 500, dtype=BF16 if i % 3 else F32) for i in range(1300)]
    if kind == "matrix":
        return [rnd(g, 33, 65), rnd(g, 64, 128, dtype=BF16)]
    return [torch.zeros(1000, device="cuda"), torch.zeros(3, device="cuda", dtype=BF16)]


def norm_of(items):
    norm = scalar(-1)
    fp8.fp8_grad_norm(items, norm, ws_of(fp8.fp8_grad_norm_workspace_bytes(items)))
    return norm


@pytest.mark.parametrize("kind", ["one", "mixed", "many", "matrix", "zero"])
@pytest.mark.parametrize("out_dt", [None, F32, BF16])
@pytest.mark.parametrize("max_norm", [0.37, 1e6])
def test_gradient_norm_and_clip(kind, out_dt, max_norm):
    grads = grad_sets(kind)
    before = [x.clone() for x in grads]
    outs = None if out_dt is None else [torch.full(x.shape, math.nan, dtype=out_dt, device="cuda") for x in grads]
    items = fp8.fp8_grad_items(grads, outs)
    norm = norm_of(items)
    want = math.sqrt(sum(float(x.to(F64).square().sum()) for x in before))
    # 32 squares in FP32 (33 u of their sum), FP64 above, half of it through the root, the rounding of the result
    assert abs(norm.item() - want) <= (17 + 2) * U * want
    assert torch.equal(norm, norm_of(items))
    fp8.fp8_grad_clip(items, norm, max_norm)
    c = np.float32(max_norm) / (np.float32(norm.item()) + np.float32(1e-6))
    c = torch.tensor(min(np.float32(1.0), c), device="cuda")
    for i, x in enumerate(before):
        got = grads[i] if outs is None else outs[i]
        assert torch.equal(got, (x.float() * c).to(got.dtype)), i
        if outs is not None:
            assert torch.equal(grads[i], x)


def test_gradient_clip_into_a_flat_bucket_leaves_the_gaps():
    sizes, g = [5, 16, 1, 1000, 8], gen(5)
    grads = [rnd(g, n, dtype=BF16) for n in sizes]
    starts = np.cumsum([0] + [-(-n // 8) * 8 for n in sizes])
    bucket = torch.full((int(starts[-1]),), 9.0, device="cuda")
    items = fp8.fp8_grad_items(grads, [bucket[a:a + n] for a, n in zip(starts, sizes)])
    norm = norm_of(items)
    fp8.fp8_grad_clip(items, norm, 0.5)
    gap = torch.ones_like(bucket, dtype=torch.bool)
    for a, n in zip(starts, sizes):
        gap[a:a + n] = False
    assert (bucket[gap] == 9.0).all()
    assert abs(float(bucket[~gap].to(F64).norm()) - 0.5) <= 0.5 * (2 * U + 1e-6 + 40 * U)


def test_gradient_norm_of_infinities_and_nan():
    x = torch.ones(100, device="cuda")
    x[50] = math.inf
    items = fp8.fp8_grad_items([x, torch.ones(9, device="cuda")])
    norm = norm_of(items)
    assert math.isinf(norm.item())
    fp8.fp8_grad_clip(items, norm, 1.0)
    assert torch.isnan(x[50]) and (x[:50] == 0).all()
    y = torch.ones(100, device="cuda")
    y[3] = math.nan
    items = fp8.fp8_grad_items([y])
    norm = norm_of(items)
    assert math.isnan(norm.item())
    fp8.fp8_grad_clip(items, norm, 1.0)
    assert torch.isnan(y).all()


# ------------------------------------------------------------------------------------------------ beyond 32 bits
def test_offsets_beyond_32_bits():
    """Tables, rows and gradients of more than 2^32 bytes (and 2^31 elements): the far end is read and written."""
    V, D, T = 600_000, 4096, 40
    table = torch.zeros((V, D), dtype=BF16, device="cuda")                       # 4.9 GB
    ids = torch.arange(V - T, V, device="cuda")
    table[V - T:] = rnd(gen(1), T, D, dtype=BF16)
    out = torch.empty((T, D), dtype=BF16, device="cuda")
    fp8.fp8_embedding_fwd(table, ids, 1.0, out)
    assert torch.equal(out, table[V - T:])
    dy = rnd(gen(2), T, D, dtype=BF16)
    table[300_000:300_010] = 5.0
    fp8.fp8_embedding_bwd(dy, ids, 2.0, table, ws_of(fp8.fp8_embedding_bwd_workspace_bytes(T, V, D)))
    assert torch.equal(table[V - T:], (dy.float() * 2).to(BF16)) and not table[:V - T].any()
    # layer norm over the same memory: V rows, the last ones looked at
    table[V - 3:] = rnd(gen(3), 3, D, dtype=BF16)
    gamma, beta = 1 + 0.1 * rnd(gen(4), D), rnd(gen(5), D)
    mean, rstd = torch.empty(V, device="cuda"), torch.empty(V, device="cuda")
    y = torch.empty_like(table)
    fp8.fp8_layernorm_fwd(table, gamma, beta, 1e-5, y, mean=mean, rstd=rstd)
    want, mu, rs, size = ln_reference(table[V - 3:], gamma, beta, float(np.float32(1e-5)))
    within(y[V - 3:], want, HALF[BF16] * want.abs() + 240 * U * size * (1 + 2 ** -7))
    assert (y[12345] == beta.to(BF16)).all()
    dg, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    y.zero_()
    y[V - 3:] = 1.0                                                              # the upstream gradient: the last rows only
    wdx, wsize, *_ = ln_backward_reference(y[V - 3:], table[V - 3:], gamma, mean[V - 3:], rstd[V - 3:])
    fp8.fp8_layernorm_bwd(y, table, gamma, mean, rstd, y, dg, db, ws_of(fp8.fp8_layernorm_bwd_workspace_bytes(V, D)))
    within(y[V - 3:], wdx, HALF[BF16] * wdx.abs() + 96 * U * wsize * (1 + 2 ** -7))
    assert not y[:V - 3].any() and (db == 3.0).all()
    # one gradient of 2.4 G elements
    flat = table.view(-1)
    flat.zero_()
    flat[-5:] = 3.0
    items = fp8.fp8_grad_items([flat])
    norm = norm_of(items)
    assert abs(norm.item() - math.sqrt(45)) <= 19 * U * math.sqrt(45)
    fp8.fp8_grad_clip(items, norm, 1.0)
    assert (flat[-5:].float() - 3 / math.sqrt(45)).abs().max() <= 2 ** -8 * 0.45 + 1e-6 and not flat[:-5].any()


# ------------------------------------------------------------------------------------------------ arguments
def test_python_side_checks():
    x, out = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.zeros((4, 64), dtype=BF16, device="cuda")
    one, gb = scalar(1), torch.zeros(64, device="cuda")
    for bad in (
        lambda: fp8.fp8_layernorm_fwd(x.float(), gb, gb, 1e-5, out),
        lambda: fp8.fp8_layernorm_fwd(x, gb[:32], gb, 1e-5, out),
        lambda: fp8.fp8_layernorm_fwd(x, gb, gb, 1e-5, out[:2]),
        lambda: fp8.fp8_layernorm_fwd(x.cpu(), gb, gb, 1e-5, out),
        lambda: fp8.fp8_layernorm_fwd(x.t(), gb, gb, 1e-5, out),
        lambda: fp8.fp8_layernorm_fwd(torch.zeros((4, 128), dtype=BF16, device="cuda")[:, ::2], gb, gb, 1e-5, out),
        lambda: fp8.fp8_embedding_fwd(x, torch.zeros(4, device="cuda"), 1.0, out),
        lambda: fp8.fp8_embedding_fwd(x, torch.zeros(3, device="cuda", dtype=torch.int32), 1.0, out),
        lambda: fp8.fp8_embedding_fwd(x.half(), torch.zeros(4, device="cuda", dtype=torch.int32), 1.0, out),
        lambda: fp8.fp8_grad_items([]),
        lambda: fp8.fp8_grad_items([gb], [gb, gb]),
        lambda: fp8.fp8_grad_items([gb], [gb[:32]]),
        lambda: fp8.fp8_grad_items([gb, gb.half()]),
        lambda: fp8.fp8_grad_items([gb, gb], [gb, gb.double()]),
        lambda: fp8.fp8_grad_items([gb, gb.cpu()]),
        lambda: fp8.fp8_grad_items([gb[:32], gb[:32]], [gb[:32], gb[::2]]),
        lambda: fp8.fp8_grad_items([gb[::2]]),
        lambda: fp8.fp8_grad_norm(fp8.fp8_grad_items([gb]), one.half(), ws_of(256)),
    ):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(fp8.Fp8Error):
        fp8.fp8_grad_clip(fp8.fp8_grad_items([gb]), one, 0.0)
    with pytest.raises(fp8.Fp8Error):
        fp8.fp8_layernorm_bwd(x, x, gb, gb[:4], gb[:4], out, gb, gb, ws_of(256))


# ------------------------------------------------------------------------------------------------ together
def test_calls_go_to_the_given_stream_and_into_a_graph():
    """The operators one after the other on a side stream, eagerly and as a captured graph that is replayed on new inputs."""
    T, V, D, E, k = 300, 500, 256, 8, 2
    g = gen(31)
    table, ids = rnd(g, V, D, std=0.02, dtype=BF16), token_ids(g, T, V)
    gamma, beta = 1 + 0.1 * rnd(g, D), 0.1 * rnd(g, D)
    logits, dout = rnd(g, T, E), rnd(g, T, D, dtype=BF16)
    x, y, dx = (torch.empty((T, D), dtype=BF16, device="cuda") for _ in range(3))
    mean, rstd, dg, db = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    a = scalar(0)
    dtable, norm = torch.empty((V, D), device="cuda"), scalar(0)
    r = route_outputs(T, E, k)
    dl = torch.empty((T, E), device="cuda")
    items = fp8.fp8_grad_items([dtable, dg, db])
    w = [ws_of(n) for n in (fp8.fp8_layernorm_bwd_workspace_bytes(T, D), fp8.fp8_embedding_bwd_workspace_bytes(T, V, D),
                            fp8.fp8_moe_route_workspace_bytes(T, E), fp8.fp8_grad_norm_workspace_bytes(items))]

    def step(stream=None):
        s = dict(stream=stream)
        fp8.fp8_embedding_fwd(table, ids, 50.0, x, a, **s)
        fp8.fp8_layernorm_fwd(x, gamma, beta, 1e-5, y, mean=mean, rstd=rstd, **s)
        fp8.fp8_moe_route(logits, None, True, CB, CZ, r["expert"], r["weight"], r["counts"], r["offsets"], r["rows"], r["n_routed"],
                          r["loss"], w[2], **s)
        fp8.fp8_moe_route_bwd(logits, r["expert"], r["counts"], r["n_routed"], True, CB, CZ, None, None, dl, **s)
        fp8.fp8_layernorm_bwd(dout, x, gamma, mean, rstd, dx, dg, db, w[0], **s)
        fp8.fp8_embedding_bwd(dx, ids, 50.0, dtable, w[1], **s)
        fp8.fp8_grad_norm(items, norm, w[3], **s)
        fp8.fp8_grad_clip(items, norm, 0.1, **s)

    outputs = [x, a, y, mean, rstd, dx, dg, db, dtable, norm, dl, *r.values()]
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    side = torch.cuda.Stream()
    for t in outputs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(t, v) for t, v in zip(outputs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ids.copy_(token_ids(gen(32), T, V))
    logits.copy_(rnd(gen(33), T, E))
    step()
    torch.cuda.synchronize()
    want2 = [t.clone() for t in outputs]
    assert not torch.equal(want2[0], want[0])
    for _ in range(2):
        for t in outputs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, v) for t, v in zip(outputs, want2))


def test_calls_on_one_workspace_in_order_and_on_two_at_once():
    """Calls back to back on one stream may share a workspace; calls on two streams with a workspace each run at once."""
    V, D, E, k = 3000, 320, 40, 4
    sizes = [5000, 700, 9000, 33, 5000, 4737]                   # every order of the ids up to 65536, one behind the other
    g = gen(61)
    data = []
    for T in sizes:
        x = rnd(g, T, D, dtype=BF16)
        mu = x.float().mean(1)
        data.append(dict(T=T, ids=pattern(g, T, V, "zipf"), x=x, dy=rnd(g, T, D, dtype=BF16), logits=rnd(g, T, E), mean=mu,
                         rstd=(x.float() - mu[:, None]).square().mean(1).rsqrt()))
    gamma = 1 + 0.1 * rnd(g, D)
    most = max(sizes)

    def scratch():
        return [ws_of(n) for n in (max(fp8.fp8_embedding_bwd_workspace_bytes(T, V, D) for T in sizes),
                                   max(fp8.fp8_layernorm_bwd_workspace_bytes(T, D) for T in sizes),
                                   fp8.fp8_moe_route_workspace_bytes(most, E), 1 << 16)]

    def calls(d, w, stream=None):
        T = d["T"]
        dtable, dx, dg, db, norm = torch.empty((V, D), device="cuda"), torch.empty_like(d["x"]), torch.empty(D, device="cuda"), torch.empty(D, device="cuda"), scalar(0)
        r, dl = route_outputs(T, E, k), torch.empty_like(d["logits"])
        s = dict(stream=stream)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())     # the fills of the outputs
        fp8.fp8_embedding_bwd(d["dy"], d["ids"], 1.5, dtable, w[0], **s)
        fp8.fp8_layernorm_bwd(d["dy"], d["x"], gamma, d["mean"], d["rstd"], dx, dg, db, w[1], **s)
        fp8.fp8_moe_route(d["logits"], None, True, CB, CZ, r["expert"], r["weight"], r["counts"], r["offsets"], r["rows"],
                          r["n_routed"], r["loss"], w[2], **s)
        fp8.fp8_moe_route_bwd(d["logits"], r["expert"], r["counts"], r["n_routed"], True, CB, CZ, None, None, dl, **s)
        items = fp8.fp8_grad_items([dtable, dg, db])
        fp8.fp8_grad_norm(items, norm, w[3], **s)
        fp8.fp8_grad_clip(items, norm, 0.7, **s)
        return [dtable, dx, dg, db, norm, dl, *r.values()]

    want = []
    for d in data:
        want.append(calls(d, scratch()))
        torch.cuda.synchronize()
    w = scratch()
    got = [calls(d, w) for d in data]                            # nothing waits between them
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o, v in zip(got, want) for a, b in zip(o, v))
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [scratch(), scratch()]
    got = [calls(d, ws[i % 2], streams[i % 2]) for i, d in enumerate(data)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o, v in zip(got, want) for a, b in zip(o, v))


def test_a_training_step_around_the_fp8_products():
    """Token ids to clipped gradients through the package's own calls: embedding with codes, FP8 linear layer, layer norm with
    residual, its backward, the linear layer's gradients, the table's gradient, norm and clip; the gradients against a 64-bit
    evaluation that takes the package's FP8 operands as they are."""
    T, V, D = 96, 200, 128
    g = gen(41)
    table, ids = rnd(g, V, D, std=0.02, dtype=BF16), torch.randint(0, V, (T,), generator=g, device="cuda")
    gamma, beta, w = 1 + 0.1 * rnd(g, D), 0.1 * rnd(g, D), rnd(g, D, D, std=D ** -0.5, dtype=BF16)
    dout = rnd(g, T, D, std=1e-2, dtype=BF16)
    e8 = lambda t: torch.empty(t.shape, dtype=torch.uint8, device="cuda")
    eb = lambda *s: torch.empty(s, dtype=BF16, device="cuda")
    x, y, out, dy, dxl = (eb(T, D) for _ in range(5))
    x8, w8, dy8 = e8(x), e8(w), e8(x)
    xs, a = scalar(64.0), scalar(0)
    xsi = scalar(1.0 / 64.0)
    ws_, wsi, ds_, dsi = (scalar(0) for _ in range(4))
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dw, dg, db, dtable, norm = torch.empty((D, D), device="cuda"), torch.empty(D, device="cuda"), torch.empty(D, device="cuda"), torch.empty((V, D), device="cuda"), scalar(0)
    fp8.fp8_embedding_fwd_q(table, ids, 50.0, xs, fp8.E4M3, x, x8, a)
    fp8.fp8_quantize(w, fp8.E4M3, w8, None, a, ws_, wsi)
    fp8.fp8_linear_fwd(x8, w8, xsi, wsi, y)
    fp8.fp8_layernorm_fwd(y, gamma, beta, 1e-5, out, mean=mean, rstd=rstd, residual=x)
    fp8.fp8_layernorm_bwd(dout, y, gamma, mean, rstd, dy, dg, db, ws_of(fp8.fp8_layernorm_bwd_workspace_bytes(T, D)))
    fp8.fp8_quantize(dy, fp8.E5M2, dy8, None, a, ds_, dsi)
    fp8.fp8_linear_dgrad_rm(dy8, w8, dsi, wsi, dxl)
    fp8.fp8_linear_wgrad_rm(dy8, x8, dsi, xsi, dw)
    demb = (dxl.float() + dout.float()).to(BF16)                 # the linear layer's path and the residual's
    fp8.fp8_embedding_bwd(demb, ids, 50.0, dtable, ws_of(fp8.fp8_embedding_bwd_workspace_bytes(T, V, D)))
    items = fp8.fp8_grad_items([dw, dg, db, dtable])
    plain = [t.clone() for t in (dw, dg, db, dtable)]
    fp8.fp8_grad_norm(items, norm, ws_of(fp8.fp8_grad_norm_workspace_bytes(items)))
    fp8.fp8_grad_clip(items, norm, 1.0)
    assert fp8.fp8_device_status() == 0
    # 64 bits
    xd = table[ids].to(F64) * 50.0
    x8d, w8d = x8.view(torch.float8_e4m3fn).to(F64) / 64.0, w8.view(torch.float8_e4m3fn).to(F64) * wsi.item()
    want, mu, rs, _ = ln_reference(y, gamma, beta, 1e-5, x)
    assert float((x.to(F64) - xd).norm() / xd.norm()) <= HALF[BF16]
    assert float((out.to(F64) - want).norm() / want.norm()) <= HALF[BF16]
    yd = x8d @ w8d.T
    assert float((y.to(F64) - yd).norm() / yd.norm()) <= HALF[BF16]
    dyd, _, dgd, _, dbd, _ = ln_backward_reference(dout, y, gamma, mu, rs)
    dy8d = dy8.view(torch.float8_e5m2).to(F64) * dsi.item()
    assert float((dy8d - dyd).norm() / dyd.norm()) <= 2.0 ** -3 + 2 * HALF[BF16]        # half a step of E5M2
    dembd = dy8d @ w8d + dout.to(F64)
    dtd = torch.zeros((V, D), dtype=F64, device="cuda").index_add_(0, ids, dembd) * 50.0
    wants = [dy8d.T @ x8d, dgd, dbd, dtd]
    for got, ref, h in zip(plain, wants, (2.0 ** -19, 2.0 ** -18, 2.0 ** -18, 3 * HALF[BF16])):
        assert float((got.to(F64) - ref).norm() / ref.norm()) <= h
    total = math.sqrt(sum(float(t.to(F64).square().sum()) for t in plain))
    assert abs(norm.item() - total) <= 19 * U * total
    c = min(np.float32(1.0), np.float32(1.0) / (np.float32(norm.item()) + np.float32(1e-6)))
    assert c < 1
    for got, ref in zip((dw, dg, db, dtable), plain):
        assert torch.equal(got, ref * torch.tensor(c, device="cuda"))


# ------------------------------------------------------------------------------------------------ router: exponentials, sizes
@pytest.mark.parametrize("T,E", [(150, 2), (150, 8), (300, 40), (5000, 8), (13000, 16)])      # a warp per token in one launch and two; a lane
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("normalize", [False, True])
def test_router_probabilities_far_below_the_largest(T, E, dt, normalize):
    """A token's probabilities keep the digits of FP32 however small they are: logits 0 and -x, x up to 80."""
    k = 2
    logits = torch.full((T, E), -math.inf, device="cuda", dtype=dt)
    x = torch.linspace(1.0, 80.0, T, device="cuda").to(dt)
    logits[:, 0], logits[:, 1] = 0.0, -x
    o = route(logits, None, k, normalize, 0.0, 0.0)
    assert (o["expert"][:, 0] == 0).all() and (o["expert"][:, 1] == 1).all()
    want = torch.softmax(torch.stack([torch.zeros_like(x), -x], 1).to(F64), 1)
    # The difference from the maximum is exact here.  An exponential: 2^-22 = 4 u of the hardware's exp2, u for the product with
    # the correction, 0.05 u x for the constants in it; their sum: 5 u and u; the reciprocal and the product: u each
    within(o["weight"], want, (13 + 0.05 * x.to(F64)[:, None]) * U * want)


@pytest.mark.parametrize("T,E,k", [(40, 10, 3), (300, 160, 6), (9001, 8, 2), (33001, 16, 4)])
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dloss", [math.nan, math.inf])
def test_router_gradient_of_unrouted_rows_is_zero_whatever_the_loss(T, E, k, normalize, dloss):
    logits = rnd(gen(T + E), T, E)
    logits[::7] = -math.inf
    o = route(logits, None, k, normalize, CB, CZ)
    dl = torch.full_like(logits, 3.0)
    fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], normalize, CB, CZ, scalar(dloss), torch.ones((T, k), device="cuda"), dl)
    assert (dl[::7] == 0).all() and torch.isnan(dl[1::7]).any()


@pytest.mark.parametrize("T,E,k", [(9001, 8, 2), (33001, 16, 4), (33001, 13, 4), (300, 160, 6), (224, 256, 8), (5001, 64, 3)])
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_router_broken_rows_in_every_form(T, E, k, normalize, dt):
    """Rows with NaN or +inf: no expert, NaN weights, losses and row of the gradient; the others are as without them."""
    g = gen(T + E + 1)
    logits = rnd(g, T, E, dtype=dt)
    bad = torch.tensor([0, 7, T // 2, T - 1], device="cuda")
    logits[bad, torch.tensor([E - 1, 2, 0, E // 2], device="cuda")] = torch.tensor([math.nan, math.inf, math.inf, math.nan], device="cuda", dtype=dt)
    r = route_reference(logits, None, k, normalize, CB, CZ)
    o = route(logits, None, k, normalize, CB, CZ)
    for name in ("expert", "counts", "offsets", "rows"):
        assert torch.equal(o[name], r[name]), name
    whole = torch.ones(T, dtype=torch.bool, device="cuda")
    whole[bad] = False
    assert o["n_routed"].item() == T == r["n"]
    assert torch.isnan(o["weight"][bad]).all() and torch.isnan(o["loss"]).all()
    # as in test_router_forward_and_gradient
    rel = (4 * logits[whole].float().abs().max().item() + E / 8 + 24) * U
    within(o["weight"][whole], r["weight"][whole], rel * r["weight"][whole] + 1e-37)
    dweight, dl = rnd(g, T, k), torch.zeros_like(logits)
    fp8.fp8_moe_route_bwd(logits, o["expert"], o["counts"], o["n_routed"], normalize, CB, CZ, None, dweight, dl)
    assert torch.isnan(dl[bad]).all()
    p, idx, dw = r["p"][whole], r["expert"][whole].long(), dweight[whole].to(F64)
    u = (CB * E * r["counts"].to(F64) / (k * T * T)).expand(int(whole.sum()), E).clone()
    if not normalize:
        u.scatter_add_(1, idx, dw)
    zterm = CZ * 2 / T * r["lse"][whole][:, None] * p
    want = p * (u - (u * p).sum(1, keepdim=True)) + zterm
    size = p * (u.abs() + (u.abs() * p).sum(1, keepdim=True)) + zterm.abs()
    if normalize:
        w = r["weight"][whole]
        want.scatter_add_(1, idx, w * (dw - (dw * w).sum(1, keepdim=True)))
        size.scatter_add_(1, idx, w * (dw.abs() + (dw.abs() * w).sum(1, keepdim=True)))
    within(dl[whole], want, HALF[dt] * want.abs() + (4 * rel + (E + 32) * U) * size + 1e-37)


@pytest.mark.parametrize("T,E,k", [(100003, 8, 2), (400001, 8, 2), (400001, 13, 3), (200003, 72, 2)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_router_of_many_tokens(T, E, k, dt):
    """More tokens than one turn of all lanes takes, forward and backward."""
    for normalize, with_bias in ((True, True), (False, False)):
        test_router_forward_and_gradient(T, E, k, dt, normalize, with_bias)


# ------------------------------------------------------------------------------------------------ layer norm: rows one after the other
LONG_ROWS = [(1000, 4104), (1100, 5120), (700, 8192), (700, 8200), (600, 12288), (600, 12296), (500, 16384)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,D", LONG_ROWS)
def test_layernorm_forward_of_long_rows_one_after_the_other(T, D, residual):
    """Rows above 4096 columns, several to a CTA: more than it keeps on the way, and not the same number for each."""
    test_layernorm_forward(T, D, residual)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,D", LONG_ROWS + [(5000, 8200), (9700, 4104), (5000, 6000)])
def test_layernorm_backward_of_long_rows_one_after_the_other(T, D, accumulate):
    """The same for the gradient, and more than the 32 rows of a CTA whose statistics travel together."""
    test_layernorm_backward(T, D, accumulate)


# ------------------------------------------------------------------------------------------------ amax of NaN, lists of large gradients
@pytest.mark.parametrize("T", [1, 8, 300, 4200])
def test_amax_of_an_output_with_nan_is_nan(T):
    """Every way in which the amax is set to zero first: a NaN outranks all numbers and infinities."""
    D = 4096
    g, x, gamma, beta = ln_data(T, D, seed=8)
    table = rnd(g, T + 1, D, std=0.02, dtype=BF16)
    x[T - 1, 17], table[T - 1, 5], table[0, 9] = math.nan, math.nan, math.inf
    out, a = torch.empty_like(x), scalar(1e30)
    fp8.fp8_layernorm_fwd(x, gamma, beta, 1e-5, out, amax_out=a)
    assert math.isnan(a.item()) and torch.isnan(out[T - 1]).all() and torch.isfinite(out[:T - 1]).all()
    fp8.fp8_embedding_fwd(table, torch.arange(T, device="cuda"), 1.0, out, a)
    assert math.isnan(a.item())
    table[T - 1, 5] = 0.0
    fp8.fp8_embedding_fwd(table, torch.arange(T, device="cuda"), 1.0, out, a)
    assert math.isinf(a.item())


def test_gradient_norm_and_clip_of_many_large_tensors():
    """More tensors than one launch takes, each of many chunks."""
    g = gen(78)
    sizes = [100_000 + 4096 * (i % 7) + i for i in range(1100)]
    grads = [rnd(g, n, std=0.01 * (1 + i % 5), dtype=BF16 if i % 2 else F32) for i, n in enumerate(sizes)]
    outs = [torch.full((n,), math.nan, dtype=BF16 if i % 3 else F32, device="cuda") for i, n in enumerate(sizes)]
    items = fp8.fp8_grad_items(grads, outs)
    norm = norm_of(items)
    want = math.sqrt(sum(float(x.to(F64).square().sum()) for x in grads))
    assert abs(norm.item() - want) <= (17 + 2) * U * want               # as in test_gradient_norm_and_clip
    fp8.fp8_grad_clip(items, norm, 2.5)
    c = torch.tensor(np.float32(2.5) / (np.float32(norm.item()) + np.float32(1e-6)), device="cuda")
    assert c < 1
    for i, (x, o) in enumerate(zip(grads, outs)):
        assert torch.equal(o, (x.float() * c).to(o.dtype)), i


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("n", [1, 3, 4, 8, 1023, 4095, 4096, 4097, 4100, 148 * 4096 + 13, 20_000_003])
def test_gradient_clip_in_place_gives_the_bits_of_a_clip_elsewhere(n, dt):
    g = gen(n)
    x = rnd(g, n, dtype=dt)
    other = torch.full_like(x, math.nan)
    elsewhere, here = fp8.fp8_grad_items([x], [other]), fp8.fp8_grad_items([x])
    norm = norm_of(here)
    fp8.fp8_grad_clip(elsewhere, norm, 0.3)
    fp8.fp8_grad_clip(here, norm, 0.3)
    assert torch.equal(x, other)


def test_a_gradient_that_is_listed_twice_is_refused():
    """Tied weights: clipped in place, two CTAs would scale the same elements.  Empty tensors may share their address."""
    a, b, empty = torch.ones(100, device="cuda"), torch.ones(100, device="cuda"), torch.empty(0, device="cuda")
    for grads, outs in (([a, b, a], None), ([a, b], [a, a]), ([a, b.view(10, 10)], [b, b.view(10, 10)])):
        with pytest.raises(ValueError, match="twice"):
            fp8.fp8_grad_items(grads, outs)
    assert len(fp8.fp8_grad_items([a, empty, b, empty])) == 4
