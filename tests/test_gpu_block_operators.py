"""GPU parity of the operators between a block's FP8 products and of the optimizer: rotary positions on the QKV projection, the
joint of two blocks, AdamW, against plain evaluations in 64 bits.

Tolerances.  u = 2^-24 is half a step of FP32, h = eps / 2 half a step of the output's type.  A sum of n FP32 terms in any order is
off by at most n u times the sum of their magnitudes (to first order); a tree of sums by its depth.  The sums over a row here are
of at most 32 terms in a row of one thread and 9 levels above: 41 u; its reciprocal root halves that and adds 4 u (2 ulp).  The
exponential of the sigmoid is off by 2^-22 of itself plus 2 u |gate| through its rounded argument, the quotient by 4 u.  With the
few products around them every FP32 value below is off by less than 64 u of the magnitudes that went into it, (64 + 2 |gate|) u with
a sigmoid, on top of one rounding to the output's type.
"""
import decimal
import math

import numpy as np
import pytest
import torch

import paper_2505_20524_b200 as fp8

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF16, F32, F64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.uint8
NAN = math.nan


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rnd(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def scalar(v):
    return torch.full((1,), float(v), device="cuda")


def full(shape, v=7.0, dtype=BF16):
    return torch.full(shape, v, dtype=dtype, device="cuda")


def ws_of(n):
    return torch.full((n,), 0xA5, dtype=U8, device="cuda")       # scratch needs no preparation


def within(got, ref, tol):
    """|got - ref| <= tol elementwise (all in 64 bits); the message names the worst element."""
    d = (got.to(F64) - ref).abs() - tol
    assert not torch.isnan(d).any()
    worst = int(d.argmax())
    assert d.max() <= 0, (worst, got.reshape(-1)[worst].item(), ref.reshape(-1)[worst].item(), tol.reshape(-1)[worst].item())


def codes_of(x, scale, fmt):
    x = x.contiguous()
    out8 = torch.empty(x.shape, dtype=U8, device="cuda")
    if x.numel():
        fp8.fp8_cast(x.reshape(-1), scale, fmt, out8.reshape(-1))    # flat: any length
    return out8


def amax_of(x):
    return x.float().abs().max().item() if x.numel() else 0.0


# ------------------------------------------------------------------------------------------------ table
def frequencies(rot, base, kind, factor, length, low, high):
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if kind == fp8.ROPE_LINEAR:
        f = [x / factor for x in f]
    if kind == fp8.ROPE_NTK:
        wide = base * factor ** (rot / (rot - 2.0))
        f = [wide ** (-2.0 * i / rot) for i in range(rot // 2)]
    if kind == fp8.ROPE_BY_PARTS:
        w = [min(1.0, max(0.0, (length * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [(1 - a) * x / factor + a * x for a, x in zip(w, f)]
    return torch.tensor(f, dtype=F64, device="cuda")


@pytest.mark.parametrize("N,rot,kind", [(1, 16, fp8.ROPE_PLAIN), (7, 16, fp8.ROPE_NTK), (1000, 64, fp8.ROPE_PLAIN),
                                        (1000, 80, fp8.ROPE_LINEAR), (4097, 128, fp8.ROPE_BY_PARTS), (300, 256, fp8.ROPE_BY_PARTS),
                                        (1 << 20, 32, fp8.ROPE_NTK)])
@pytest.mark.parametrize("magnitude", [1.0, 1.277])
def test_rope_table(N, rot, kind, magnitude):
    base, factor, length, low, high = 10000.0, 8.0, 2048.0, 1.0, 32.0
    cos, sin = full((N, rot // 2), NAN, F32), full((N, rot // 2), NAN, F32)
    fp8.fp8_rope_table(cos, sin, base, kind, factor, length, low, high, magnitude)
    angle = torch.arange(N, device="cuda", dtype=F64)[:, None] * frequencies(rot, base, kind, factor, length, low, high)
    # 2 ulp (4 u) of the function, u of the rounded rest, u of the product; the angle is off by a few 2^-53 of itself on either side
    for got, ref in ((cos, angle.cos()), (sin, angle.sin())):
        within(got, ref * magnitude, (6 * U * ref.abs() + 8 * 2.0 ** -53 * angle) * magnitude)
    assert (cos[0] == np.float32(magnitude)).all() and (sin[0] == 0).all()


def exact_turns(rot, base, kind=fp8.ROPE_PLAIN, factor=1.0, length=1.0, low=0.0, high=1.0, bits=160):
    """Turns per position of each pair, times 2^bits, as whole numbers: from decimals of 80 digits."""
    with decimal.localcontext() as ctx:
        ctx.prec = 80
        D = decimal.Decimal
        full_turn = 2 * D("3.1415926535897932384626433832795028841971693993751058209749445923078164062862090")
        out = []
        for i in range(rot // 2):
            b = D(base) * D(factor) ** (D(rot) / (rot - 2)) if kind == fp8.ROPE_NTK else D(base)
            f = b ** (D(-2 * i) / rot)
            if kind == fp8.ROPE_LINEAR:
                f /= D(factor)
            if kind == fp8.ROPE_BY_PARTS:
                w = min(D(1), max(D(0), (D(length) * f / full_turn - D(low)) / (D(high) - D(low))))
                f = (1 - w) * f / D(factor) + w * f
            out.append(int((f / full_turn * 2 ** bits).to_integral_value()))
        return out


def exact_cos_sin(turns, pos, bits=160):
    """cos and sin of a position's angle: what is left of it next to the nearest quarter turn is exact before it becomes a float."""
    quarter = 1 << (bits - 2)
    k = (turns * pos + quarter // 2) // quarter
    x = (turns * pos - k * quarter) / (1 << bits) * (2 * math.pi)
    c, s = math.cos(x), math.sin(x)
    return ((c, s), (-s, c), (-c, -s), (s, -c))[k % 4]


# numerators of fractions next to pi and its half: a sine or a cosine next to 0 at frequency 1
NEAR_ZEROS = [11, 22, 333, 344, 355, 51819, 52174, 103993, 104348, 208341, 312689, 573204, 833719, 1146408, 4272943, 5419351, 80143857]


@pytest.mark.parametrize("N,rot,base,kind,factor", [
    (131072, 128, 500000.0, fp8.ROPE_BY_PARTS, 16.0), (1 << 21, 64, 10000.0, fp8.ROPE_PLAIN, 1.0), (80143858, 16, 10000.0, fp8.ROPE_PLAIN, 1.0),
    (1 << 20, 32, 10000.0, fp8.ROPE_NTK, 8.0), (1 << 19, 256, 10000.0, fp8.ROPE_LINEAR, 7.0),
    (8192, 64, 2.0 ** -20, fp8.ROPE_PLAIN, 1.0), (1 << 20, 16, 1.0, fp8.ROPE_LINEAR, 2.0 ** -13)])   # many turns per position
def test_rope_table_to_two_ulp(N, rot, base, kind, factor):
    """Entries next to the zeros of both functions and far out, against angles in 160 bits."""
    half = rot // 2
    cos, sin = full((N, half), NAN, F32), full((N, half), NAN, F32)
    fp8.fp8_rope_table(cos, sin, base, kind, factor, 8192.0, 1.0, 32.0)
    turns = exact_turns(rot, base, kind, factor, 8192.0, 1.0, 32.0)
    rng = np.random.default_rng(N + rot)
    rows = sorted({x for x in NEAR_ZEROS if x < N} | {int(x) for x in rng.integers(0, N, 300)} | {0, N - 1})
    # and where the table itself is smallest
    for t in (cos, sin):
        rows += t[1:].abs().amin(1).topk(min(100, N - 1), largest=False).indices.add(1).tolist()
    at = torch.tensor(rows, device="cuda")
    want = np.array([[exact_cos_sin(f, r) for f in turns] for r in rows])
    for j, table in enumerate((cos, sin)):
        ref, got = want[..., j], table[at].cpu().numpy().astype(np.float64)
        ulp = np.ldexp(1.0, np.frexp(ref)[1] - 24)
        ulp[ref == 0] = 0.0
        off = np.abs(got - ref) - 2 * ulp
        worst = np.unravel_index(off.argmax(), off.shape)
        assert off.max() <= 0, (rows[worst[0]], worst[1], got[worst], ref[worst], (np.abs(got - ref) / np.maximum(ulp, 1e-300)).max())


# ------------------------------------------------------------------------------------------------ rotary positions
class RopeCase:
    def __init__(self, T, Hq, Hkv, d, rot, mode, interleaved, positions, N=None, strided=False, seed=0):
        g = gen(1000 * T + 10 * d + rot + seed)
        self.T, self.Hq, self.Hkv, self.d, self.rot, self.mode, self.interleaved = T, Hq, Hkv, d, rot, mode, interleaved
        self.N = N or max(3, T // 2)
        self.W = (Hq + 2 * Hkv) * d
        self.alpha, self.eps = 0.6, 1e-6
        self.qkv = rnd(g, T, self.W + (24 if strided else 0), dtype=BF16)[:, :self.W]
        self.cos = self.sin = None
        if rot:
            a = torch.rand((self.N, rot // 2), generator=g, device="cuda") * 6.3
            self.cos, self.sin = (1.1 * a.cos()).contiguous(), (1.1 * a.sin()).contiguous()
        self.pos = None
        if positions is not None:
            self.pos = torch.randint(0, self.N, (T,), generator=g, device="cuda", dtype=positions)
            if T > 4:
                self.pos[T // 2], self.pos[T // 3], self.pos[1] = -1, self.N, -(1 << 31)
                for t in (T // 2, T // 3, 1):
                    self.qkv[t] = NAN                                  # padding: whatever it holds
        self.dq, self.dk, self.dv = (rnd(g, T, H, d, dtype=BF16) for H in (Hq, Hkv, Hkv))
        self.how = (mode, self.alpha, self.eps, self.cos, self.sin, self.pos, interleaved)

    def known(self):
        if self.pos is None or not self.rot:
            return torch.ones(self.T, dtype=torch.bool, device="cuda")
        return (self.pos >= 0) & (self.pos < self.N)

    def turn(self, x, sign, size=False):
        """The rotation (sign -1: back) of [T, H, d] in 64 bits; size: of the magnitudes."""
        if not self.rot:
            return x
        pos = self.pos.long() if self.pos is not None else torch.arange(self.T, device="cuda") % self.N
        at = torch.where(self.known(), pos, 0)
        c, s = self.cos[at].to(F64)[:, None], self.sin[at].to(F64)[:, None] * sign
        if size:
            c, s = c.abs(), -s.abs()
        r = self.rot
        i, j = (slice(0, r, 2), slice(1, r, 2)) if self.interleaved else (slice(0, r // 2), slice(r // 2, r))
        out = x.clone()
        out[..., i] = x[..., i] * c - x[..., j] * s
        out[..., j] = x[..., j] * c + (x[..., i] * s if not size else -x[..., i] * s)
        return out

    def heads(self):
        x = torch.where(self.known()[:, None], self.qkv.to(F64), 0.0)
        return x.view(self.T, -1, self.d).split([self.Hq + self.Hkv, self.Hkv], 1)

    def regular(self, x):
        if self.mode == fp8.QK_RMS:
            return x * (x.square().mean(-1, keepdim=True) + float(np.float32(self.eps))).rsqrt()
        return torch.tanh(float(np.float32(self.alpha)) * x) if self.mode == fp8.QK_TANH else x

    def forward(self):
        """(reference, magnitudes) of the rows' heads."""
        x, v = self.heads()
        y = self.regular(x)
        keep = self.known()[:, None, None]
        return torch.cat([self.turn(y, 1.0), v], 1) * keep, torch.cat([self.turn(y.abs(), 1.0, True), v.abs()], 1)

    def backward(self):
        x, _ = self.heads()
        do = torch.cat([self.dq, self.dk], 1).to(F64)
        u, size = self.turn(do, -1.0), self.turn(do.abs(), -1.0, True)
        if self.mode == fp8.QK_RMS:
            r = (x.square().mean(-1, keepdim=True) + float(np.float32(self.eps))).rsqrt()
            xh = x * r
            u, size = r * (u - xh * (u * xh).mean(-1, keepdim=True)), r * (size + xh.abs() * (size * xh.abs()).mean(-1, keepdim=True))
        elif self.mode == fp8.QK_TANH:
            a = float(np.float32(self.alpha))
            slope = a / torch.cosh(a * x).square()
            u, size = u * slope, size * slope * (1 + (a * x).abs() / 16)     # the exponential's rounded argument
        dv = self.dv.to(F64)
        keep = self.known()[:, None, None]
        return torch.cat([u, dv], 1) * keep, torch.cat([size, dv.abs()], 1)


ROPE_CASES = [  # T, Hq, Hkv, d, rot, positions, strided
    (1, 1, 1, 16, 16, None, False), (1, 32, 8, 128, 128, torch.int64, False), (3, 5, 1, 64, 32, None, True),
    (33, 4, 4, 64, 64, torch.int32, True), (257, 32, 8, 128, 128, None, False), (100, 3, 3, 80, 80, torch.int64, False),
    (77, 6, 2, 96, 48, torch.int32, False), (50, 7, 1, 192, 64, None, True), (40, 8, 2, 256, 256, torch.int64, False),
    (65, 2, 2, 32, 16, None, False), (31, 9, 0, 128, 64, torch.int32, True), (20, 5, 5, 112, 0, None, False),
    (9, 130, 33, 256, 32, None, False),
    (11, 130, 33, 256, 256, torch.int64, True), (700, 70, 10, 128, 128, torch.int32, False), (3000, 1, 1, 16, 16, torch.int64, False),
    (6000, 2, 1, 64, 64, torch.int32, True),
]


@pytest.mark.parametrize("T,Hq,Hkv,d,rot,positions,strided", ROPE_CASES)
@pytest.mark.parametrize("mode", [fp8.QK_RMS, fp8.QK_TANH, fp8.QK_NONE])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_forward(T, Hq, Hkv, d, rot, positions, strided, mode, interleaved):
    c = RopeCase(T, Hq, Hkv, d, rot, mode, interleaved, positions, strided=strided)
    q, k, v = (full((T, H, d)) for H in (Hq, Hkv, Hkv))
    kv = (k, v) if Hkv else (None, None)
    amax = full((3,), -1.0, F32)
    fp8.fp8_rope_qkv_fwd(c.qkv, Hq, Hkv, *c.how, q, *kv, amax_out=amax)
    ref, size = c.forward()
    got = torch.cat([q, k, v], 1)
    within(got, ref, HALF[BF16] * ref.abs() + 64 * U * size)
    assert torch.equal(got[:, Hq + Hkv:], torch.where(c.known()[:, None], c.qkv, 0.0).view(T, -1, d)[:, Hq + Hkv:])
    assert (got[~c.known()] == 0).all()
    assert amax.tolist() == [amax_of(x) for x in (q, k, v)]
    for fmt in (fp8.E4M3, fp8.E5M2):
        scales = torch.tensor([30.0, 1000.0, 7.0], device="cuda")
        codes = [full(x.shape, 0xEE, U8) for x in (q, k, v)]
        outs = [full(x.shape) for x in (q, k, v)]
        a2 = full((3,), -1.0, F32)
        some = [x if i == 0 or Hkv else None for i, x in enumerate(codes)]
        others = [x if i == 0 or Hkv else None for i, x in enumerate(outs)]
        fp8.fp8_rope_qkv_fwd_q(c.qkv, Hq, Hkv, *c.how, scales, fmt, *some, *others, amax_out=a2)
        assert torch.equal(a2, amax)
        for i, x in enumerate((q, k, v)):
            assert torch.equal(outs[i], x) and torch.equal(codes[i], codes_of(x, scales[i:i + 1], fmt))
        for x in codes:
            x.fill_(0xEE)
        fp8.fp8_rope_qkv_fwd_q(c.qkv, Hq, Hkv, *c.how, scales, fmt, *some)                # codes only
        for i, x in enumerate((q, k, v)):
            assert torch.equal(codes[i], codes_of(x, scales[i:i + 1], fmt))


@pytest.mark.parametrize("d,mode", [(64, fp8.QK_RMS), (128, fp8.QK_RMS), (64, fp8.QK_NONE), (128, fp8.QK_NONE), (128, fp8.QK_TANH)])
def test_rope_forward_agrees_with_qk_norm_rope(d, mode):
    c = RopeCase(99, 8, 2, d, d, mode, False, None, N=40)
    q, k = full((99, 8, d)), full((99, 2, d))
    fp8.fp8_rope_qkv_fwd(c.qkv, 8, 2, *c.how, q, k, None)
    for got, first in ((q, 0), (k, 8)):
        x = c.qkv.view(99, -1, d)[:, first:first + got.shape[1]].contiguous()
        out = torch.empty_like(x)
        fp8.fp8_qk_norm_rope(x, mode, c.alpha, c.eps, c.cos, c.sin, c.N, out)
        # both are within 64 u of the same values in front of their rounding, which then moves them by 2 h at most
        assert ((out.to(F64) - got.to(F64)).abs() <= 2 * HALF[BF16] * out.to(F64).abs() + 128 * U * 8).all()
        assert (out != got).to(F64).mean() < 1e-2


def test_rope_leaves_out_what_is_not_asked_for():
    c = RopeCase(17, 6, 3, 64, 32, fp8.QK_RMS, True, torch.int64)
    want = [full((17, H, 64)) for H in (6, 3, 3)]
    fp8.fp8_rope_qkv_fwd(c.qkv, 6, 3, *c.how, *want)
    for only in range(3):
        outs = [full(x.shape) if i == only else None for i, x in enumerate(want)]
        amax = full((3,), -1.0, F32)
        fp8.fp8_rope_qkv_fwd(c.qkv, 6, 3, *c.how, *outs, amax_out=amax)
        assert torch.equal(outs[only], want[only]) and amax.tolist() == [amax_of(x) for x in want]


@pytest.mark.parametrize("T,Hq,Hkv,d,rot,positions,strided", ROPE_CASES)
@pytest.mark.parametrize("mode", [fp8.QK_RMS, fp8.QK_TANH, fp8.QK_NONE])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient(T, Hq, Hkv, d, rot, positions, strided, mode, interleaved):
    c = RopeCase(T, Hq, Hkv, d, rot, mode, interleaved, positions, strided=strided)
    ref, size = (x.reshape(T, -1) for x in c.backward())
    for t in c.known().logical_not().nonzero().flatten().tolist():
        c.dq[t] = NAN
    wide = full((T, c.W + 16))
    dqkv = wide[:, :c.W] if strided else full((T, c.W))
    amax = scalar(-1)
    grads = (c.dq, c.dk, c.dv) if Hkv else (c.dq, None, None)
    saved = None if mode == fp8.QK_NONE and T % 2 else c.qkv
    fp8.fp8_rope_qkv_bwd(*grads, saved, *c.how, dqkv, amax_out=amax)
    within(dqkv, ref, HALF[BF16] * ref.abs() + 64 * U * size)
    assert (dqkv[~c.known()] == 0).all() and amax.item() == amax_of(dqkv)
    assert (wide[:, c.W:] == 7).all()
    for fmt in (fp8.E5M2, fp8.E4M3):
        scale, codes, a2, again = scalar(300.0), full((T, c.W), 0xEE, U8), scalar(-1), full((T, c.W))
        fp8.fp8_rope_qkv_bwd_q(*grads, saved, *c.how, scale, fmt, codes, again, a2)
        assert torch.equal(again, dqkv) and torch.equal(codes, codes_of(dqkv, scale, fmt)) and a2.item() == amax.item()
        codes.fill_(0xEE)
        fp8.fp8_rope_qkv_bwd_q(*grads, saved, *c.how, scale, fmt, codes)
        assert torch.equal(codes, codes_of(dqkv, scale, fmt))


@pytest.mark.parametrize("mode", [fp8.QK_RMS, fp8.QK_TANH, fp8.QK_NONE])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient_against_differences(mode, interleaved):
    """The formula of the gradient against central differences of the forward's formula (64 bits, step 1e-5: 1e-9)."""
    c = RopeCase(5, 2, 1, 32, 16, mode, interleaved, None)
    ref, _ = c.backward()
    x = c.qkv.to(F64).view(5, -1, 32)
    do = torch.cat([c.dq, c.dk], 1).to(F64)
    f = lambda y: (c.turn(c.regular(y[:, :3]), 1.0) * do).sum().item() + (y[:, 3:] * c.dv.to(F64)).sum().item()  # noqa: E731
    for t, h, i in [(0, 0, 0), (1, 1, 3), (2, 2, 9), (3, 0, 15), (4, 2, 16), (4, 1, 31), (2, 3, 5)]:
        e = torch.zeros_like(x)
        e[t, h, i] = 1e-5
        assert abs((f(x + e) - f(x - e)) / 2e-5 - ref[t, h, i].item()) < 1e-7 * max(1.0, ref.abs().max().item())


def test_rope_beyond_32_bit_offsets():
    T, Hq, Hkv, d = 360000, 32, 8, 128
    qkv = torch.empty((T, 48 * d), dtype=BF16, device="cuda")                       # 2.2e9 elements
    assert qkv.numel() > 2 ** 31
    last = rnd(gen(1), 64, 48 * d, dtype=BF16)
    qkv.zero_()
    qkv[-64:] = last
    a = torch.rand((T, d // 2), generator=gen(2), device="cuda")
    cos, sin = a.cos(), a.sin()
    q, k, v = (torch.empty((T, H, d), dtype=BF16, device="cuda") for H in (Hq, Hkv, Hkv))
    how = (fp8.QK_RMS, 0.0, 1e-6)
    fp8.fp8_rope_qkv_fwd(qkv, Hq, Hkv, *how, cos, sin, None, False, q, k, v)
    want = [full((64, H, d)) for H in (Hq, Hkv, Hkv)]
    fp8.fp8_rope_qkv_fwd(last, Hq, Hkv, *how, cos[-64:].contiguous(), sin[-64:].contiguous(), None, False, *want)
    assert all(torch.equal(x[-64:], w) for x, w in zip((q, k, v), want)) and (q[:-64] == 0).all()
    out = torch.empty_like(qkv)
    fp8.fp8_rope_qkv_bwd(q, k, v, qkv, *how, cos, sin, None, False, out)
    back = full((64, 48 * d))
    fp8.fp8_rope_qkv_bwd(*want, last, *how, cos[-64:].contiguous(), sin[-64:].contiguous(), None, False, back)
    assert torch.equal(out[-64:], back)


# ------------------------------------------------------------------------------------------------ joint of two blocks
POST = [fp8.NORM_RMS, fp8.NORM_LAYERSCALE, fp8.NORM_NONE]


class JointCase:
    def __init__(self, T, D, post, gate, pre, y=True):
        g = gen(T * 31 + D + post)
        self.T, self.D, self.post, self.has_gate, self.pre, self.has_y = T, D, post, gate is not None, pre, y
        self.gate_mode = gate if gate is not None else fp8.GATE_LINEAR
        self.x = rnd(g, T, D, dtype=BF16)
        self.y = rnd(g, T, D, std=3.0, dtype=BF16) if y else None
        self.gate = rnd(g, T, D, std=2.0, dtype=BF16) if self.has_gate else None
        if self.has_gate and T > 2:
            self.gate[1, :4] = torch.tensor([80.0, -80.0, 300.0, -300.0], dtype=BF16)
        self.gq = 1 + rnd(g, D, std=0.3) if y and post != fp8.NORM_NONE else None
        self.gp = 1 + rnd(g, D, std=0.3) if pre else None
        self.a, self.b, self.eps = (0.75, -1.25, 1e-5) if y else (1.0, 0.0, 1e-5)
        self.how = (post, self.gate_mode, self.a, self.b)
        self.dout = rnd(g, T, D, std=1e-2, dtype=BF16) if pre else None
        self.dh = rnd(g, T, D, std=1e-2, dtype=BF16)

    def ins(self):
        return (self.x, self.y, self.gate, self.gq, self.gp, *self.how)

    def weight(self):
        """s, s', and the units of rounding that the sigmoid adds, in 64 bits."""
        if not self.has_gate:
            one = torch.ones((), dtype=F64, device="cuda")
            return one, one * 0, 0.0
        g = self.gate.to(F64)
        if self.gate_mode == fp8.GATE_SIGMOID:
            return torch.sigmoid(g), torch.sigmoid(g) * torch.sigmoid(-g), 2 * g.abs()
        return g, torch.ones_like(g), 0.0

    def z(self, r_post=None):
        y = self.y.to(F64)
        if self.post == fp8.NORM_RMS:
            r = (y.square().mean(1) + float(np.float32(self.eps))).rsqrt() if r_post is None else r_post.to(F64)
            y = y * r[:, None]
        return y, y * self.gq.to(F64) if self.gq is not None else y


JOINT = [(1, 8), (3, 16), (33, 72), (257, 256), (130, 264), (65, 520), (40, 1032), (300, 1600), (31, 4096), (20, 4104), (19, 8192),
         (9, 8200), (12, 16384), (1000, 128),
         (2000, 520), (1800, 2056), (1500, 8200), (1300, 12296), (5000, 512), (9001, 64), (3001, 248)]       # many rows on a CTA


@pytest.mark.parametrize("T,D", JOINT)
@pytest.mark.parametrize("post,gate,pre,y", [(p, g, r, True) for p in POST for g in (None, fp8.GATE_LINEAR, fp8.GATE_SIGMOID)
                                             for r in (False, True)] + [(fp8.NORM_NONE, None, True, False)])
def test_joint_forward_and_gradient(T, D, post, gate, pre, y):
    c = JointCase(T, D, post, gate, pre, y)
    f64 = lambda t: t.to(F64)  # noqa: E731
    h, out = full((T, D)), full((T, D)) if pre else None
    rms = y and post == fp8.NORM_RMS
    rq, rp, amax = full((T,), NAN, F32) if rms else None, full((T,), NAN, F32) if pre else None, scalar(-1)
    fp8.fp8_block_norm_fwd(*c.ins(), c.eps, h, out, r_post=rq, r_pre=rp, amax_out=amax)
    s, slope, extra = c.weight()
    ref, size = c.a * f64(c.x), (c.a * f64(c.x)).abs()
    if y:
        yh, z = c.z()
        ref, size = ref + c.b * s * z, size + (c.b * s * z).abs()
    within(h, ref, HALF[BF16] * ref.abs() + (64 + extra) * U * size)
    if rms:
        exact = (f64(c.y).square().mean(1) + float(np.float32(c.eps))).rsqrt()
        within(rq, exact, 32 * U * exact)
    last = h
    if pre:
        exact = (f64(h).square().mean(1) + float(np.float32(c.eps))).rsqrt()          # of the stored sum
        within(rp, exact, 32 * U * exact)
        want = f64(c.gp) * f64(h) * exact[:, None]
        within(out, want, (HALF[BF16] + 64 * U) * want.abs())
        last = out
    assert amax.item() == amax_of(last)
    for fmt in (fp8.E4M3, fp8.E5M2):
        h2, o2, o8, a2, scale = full((T, D)), full((T, D)) if pre else None, full((T, D), 0xEE, U8), scalar(-1), scalar(37.0)
        fp8.fp8_block_norm_fwd_q(*c.ins(), c.eps, scale, fmt, h2, o2, o8, amax_out=a2)
        assert torch.equal(h2, h) and a2.item() == amax.item() and torch.equal(o8, codes_of(last, scale, fmt))
        assert not pre or torch.equal(o2, out)
        o8.fill_(0xEE)
        fp8.fp8_block_norm_fwd_q(*c.ins(), c.eps, scale, fmt, h2 if y else None, None, o8)            # codes only
        assert torch.equal(o8, codes_of(last, scale, fmt))

    # gradient, from the forward's own h and statistics
    ones = torch.ones(T, dtype=F64, device="cuda")
    rq64, rp64 = f64(rq) if rms else ones, f64(rp) if pre else ones
    for with_dh in ([True, False] if pre else [True]):
        G = f64(c.dh) if with_dh else torch.zeros((T, D), dtype=F64, device="cuda")
        mag = G.abs()
        if pre:
            hh = f64(h) * rp64[:, None]
            e = f64(c.dout) * f64(c.gp)
            G = G + rp64[:, None] * (e - hh * (e * hh).mean(1, keepdim=True))
            mag = mag + rp64[:, None] * (e.abs() + hh.abs() * (e * hh).abs().mean(1, keepdim=True))
        dx, dy, dgate = full((T, D)), full((T, D)) if y else None, full((T, D)) if c.has_gate else None
        dgq = full((D,), 0.5, F32) if c.gq is not None else None
        dgp = full((D,), 0.25, F32) if pre else None
        ws = ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(T, D))
        args = (c.dout, c.dh if with_dh else None, h if pre else None, c.y, c.gate, c.gq, c.gp, rq, rp, *c.how)
        amax = scalar(-1)
        fp8.fp8_block_norm_bwd(*args, dx, dy, dgate, dgq, dgp, ws, accumulate=with_dh, amax_out=amax if y else None)
        within(dx, c.a * G, HALF[BF16] * (c.a * G).abs() + 64 * U * abs(c.a) * mag)
        n = T + 64                                                  # terms of a column's sum
        if pre:
            total, terms = (f64(c.dout) * hh).sum(0) + 0.25 * with_dh, (f64(c.dout) * hh).abs().sum(0) + 0.25 * with_dh
            within(dgp, total, n * U * terms)
        if y:
            yh, z = c.z(rq)
            dz, dz_mag = c.b * G * s, abs(c.b) * mag * s.abs()
            if c.has_gate:
                want = c.b * G * z * slope
                # values below FP32's normal numbers: 2^-126 at most
                within(dgate, want, HALF[BF16] * want.abs() + (64 + 2 * extra) * U * abs(c.b) * mag * z.abs() * slope + 2.0 ** -126)
            f, f_mag = (dz * f64(c.gq), dz_mag * f64(c.gq).abs()) if c.gq is not None else (dz, dz_mag)
            if c.gq is not None:
                terms = ((1 + extra) * dz_mag * yh.abs()).sum(0) + 0.5 * with_dh
                within(dgq, (dz * yh).sum(0) + 0.5 * with_dh, n * U * terms)
            if rms:
                spread = 1.0 + (extra / 64)
                f = rq64[:, None] * (f - yh * (f * yh).mean(1, keepdim=True))
                f_mag = rq64[:, None] * (f_mag * spread + yh.abs() * (f_mag * spread * yh.abs()).mean(1, keepdim=True))
            else:
                f_mag = f_mag * (1.0 + extra / 64)
            within(dy, f, HALF[BF16] * f.abs() + 64 * U * f_mag + 2.0 ** -126)
            assert amax.item() == amax_of(dy)
            # codes; results in the place of inputs
            d8, scale, dx2, a2 = full((T, D), 0xEE, U8), scalar(500.0), c.dh.clone() if with_dh else c.dout.clone(), scalar(-1)
            args2 = (dx2 if not with_dh else c.dout, dx2 if with_dh else None, *args[2:])
            g2 = c.gate.clone() if c.has_gate else None
            y2 = c.y.clone()
            args2 = (*args2[:3], y2, g2, *args2[5:])
            more = [full((D,), v, F32) if t is not None else None for v, t in ((0.5, dgq), (0.25, dgp))]
            fp8.fp8_block_norm_bwd_q(*args2, scale, fp8.E5M2, dx2, y2, d8, g2, *more, ws, accumulate=with_dh, amax_out=a2)
            assert torch.equal(dx2, dx) and torch.equal(y2, dy) and torch.equal(d8, codes_of(dy, scale, fp8.E5M2))
            assert a2.item() == amax.item() and (not c.has_gate or torch.equal(g2, dgate))
            assert all(t is None or torch.equal(t, w) for t, w in zip(more, (dgq, dgp)))
            d8.fill_(0xEE)
            more = [full((D,), v, F32) if t is not None else None for v, t in ((0.5, dgq), (0.25, dgp))]
            fp8.fp8_block_norm_bwd_q(*args, scale, fp8.E4M3, dx2, None, d8, g2, *more, ws, accumulate=with_dh)
            assert torch.equal(d8, codes_of(dy, scale, fp8.E4M3))


def joint_value(c, x, y, gate, gq, gp):
    """The joint in 64 bits without the rounding of h, for differences."""
    eps = float(np.float32(c.eps))
    z = y
    if c.post == fp8.NORM_RMS:
        z = z * (z.square().mean(1, keepdim=True) + eps).rsqrt()
    if gq is not None:
        z = z * gq
    if gate is not None:
        z = z * (torch.sigmoid(gate) if c.gate_mode == fp8.GATE_SIGMOID else gate)
    h = c.a * x + c.b * z
    return h, h * (h.square().mean(1, keepdim=True) + eps).rsqrt() * gp


@pytest.mark.parametrize("post", POST)
@pytest.mark.parametrize("gate", [fp8.GATE_LINEAR, fp8.GATE_SIGMOID])
def test_joint_gradient_against_differences(post, gate):
    """All gradients of the call along random directions against central differences in 64 bits.  The call's h and outputs are
    rounded to BF16: each of its directional sums of n terms is off by at most 3 h (of h, through both norms, and of the result)
    of the sum of magnitudes; the differences by 1e-8 of it."""
    c = JointCase(6, 136, post, gate, True)
    c.gate.clamp_(-8, 8)
    h, out, rq, rp = full((6, 136)), full((6, 136)), full((6,), 0, F32), full((6,), 0, F32)
    fp8.fp8_block_norm_fwd(*c.ins(), c.eps, h, out, r_post=rq if post == fp8.NORM_RMS else None, r_pre=rp)
    dx, dy, dg = (full((6, 136)) for _ in range(3))
    dgq = full((136,), 0, F32) if c.gq is not None else None
    dgp = full((136,), 0, F32)
    fp8.fp8_block_norm_bwd(c.dout, c.dh, h, c.y, c.gate, c.gq, c.gp, rq if post == fp8.NORM_RMS else None, rp, *c.how, dx, dy, dg, dgq,
                           dgp, ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(6, 136)))
    at = [None if t is None else t.to(F64) for t in (c.x, c.y, c.gate, c.gq, c.gp)]

    def loss(v):
        a, b = joint_value(c, *v)
        return ((a * c.dh.to(F64)).sum() + (b * c.dout.to(F64)).sum()).item()

    g = gen(5)
    for i, grad in enumerate((dx, dy, dg, dgq, dgp)):
        if grad is None:
            continue
        for _ in range(3):
            way = torch.randn(at[i].shape, generator=g, device="cuda", dtype=F64)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-5 * way, at[i] - 1e-5 * way
            want = (loss(up) - loss(down)) / 2e-5
            assert abs((grad.to(F64) * way).sum().item() - want) <= 3 * HALF[BF16] * (grad.to(F64) * way).abs().sum().item()


@pytest.mark.parametrize("T,D", [(5, 64), (300, 1600), (700, 4096), (300, 16384)])
@pytest.mark.parametrize("place", ["x", "y"])
def test_joint_sum_in_the_place_of_an_input(T, D, place):
    c = JointCase(T, D, fp8.NORM_RMS, fp8.GATE_SIGMOID, True)
    h, out, o2 = full((T, D)), full((T, D)), full((T, D))
    fp8.fp8_block_norm_fwd(*c.ins(), c.eps, h, out)
    x, y = c.x.clone(), c.y.clone()
    at = x if place == "x" else y
    fp8.fp8_block_norm_fwd(x, y, *c.ins()[2:], c.eps, at, o2)
    assert torch.equal(at, h) and torch.equal(o2, out)


@pytest.mark.parametrize("T,D", [(7, 16384), (8, 12288), (9, 8192), (16, 4096), (20, 4096), (150, 1032), (33, 64), (257, 256), (529, 256), (8200, 2056)])
def test_joint_amax_in_every_kind_of_grid(T, D):
    """One CTA, one cluster, a memset in front, a kernel beside: NaN and stale values too."""
    x = rnd(gen(T), T, D, dtype=BF16)
    g = torch.ones(D, device="cuda")
    for bad in (None, math.inf, NAN):
        if bad is not None:
            x[T // 2, D // 3] = bad
        h, amax = full((T, D)), scalar(1e30)
        fp8.fp8_block_norm_fwd(x, x, None, g, None, fp8.NORM_LAYERSCALE, 0, 1.0, 0.5, 0.0, h, None, amax_out=amax)
        assert amax.item() == amax_of(h) if bad is None else math.isinf(amax.item()) if math.isinf(bad) else math.isnan(amax.item())
    c = RopeCase(T, 4, 2, 64, 64, fp8.QK_NONE, False, None)
    for bad in (None, NAN):
        if bad is not None:
            c.qkv[T // 2, 4 * 64] = bad
        q, k, v, amax = full((T, 4, 64)), full((T, 2, 64)), full((T, 2, 64)), full((3,), 1e30, F32)
        fp8.fp8_rope_qkv_fwd(c.qkv, 4, 2, *c.how, q, k, v, amax_out=amax)
        assert amax[0].item() == amax_of(q) and amax[2].item() == amax_of(v)
        assert math.isnan(amax[1].item()) if bad is not None else amax[1].item() == amax_of(k)


@pytest.mark.parametrize("T,D", [(1, 16384), (3, 12296), (8, 8200), (5, 4096), (16, 8), (2, 1032)])
def test_joint_gradient_of_few_rows_without_sums(T, D):
    """No gammas: the amax takes the other way, a cluster of a few large CTAs among them."""
    c = JointCase(T, D, fp8.NORM_NONE, fp8.GATE_LINEAR, False)
    dx, dy, dg, amax = full((T, D)), full((T, D)), full((T, D)), scalar(9e9)
    ws = ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(T, D))
    fp8.fp8_block_norm_bwd(None, c.dh, None, c.y, c.gate, None, None, None, None, *c.how, dx, dy, dg, None, None, ws, amax_out=amax)
    G = c.dh.to(F64)
    within(dy, c.b * G * c.gate.to(F64), (HALF[BF16] + 8 * U) * (c.b * G * c.gate.to(F64)).abs() + 2.0 ** -126)
    within(dg, c.b * G * c.y.to(F64), (HALF[BF16] + 8 * U) * (c.b * G * c.y.to(F64)).abs() + 2.0 ** -126)
    assert amax.item() == amax_of(dy)


def test_two_streams_at_once():
    """Calls side by side, each with its own outputs, workspace and step."""
    g1, g2 = torch.cuda.Stream(), torch.cuda.Stream()
    cases = [(RopeCase(3000, 8, 2, 128, 128, fp8.QK_RMS, False, None), JointCase(2000, 2048, fp8.NORM_RMS, None, True),
              AdamCase([300001, 77, 4096], 8, BF16, seed=s)) for s in (1, 2)]
    outs = []
    for (c, j, a), stream in zip(cases, (g1, g2)):
        q, k, v, dqkv = full((3000, 8, 128)), full((3000, 2, 128)), full((3000, 2, 128)), full((3000, c.W))
        h, out, dx, dy = (full((2000, 2048)) for _ in range(4))
        rq, rp, dgq, dgp, am = full((2000,), 0, F32), full((2000,), 0, F32), full((2048,), 0, F32), full((2048,), 0, F32), scalar(0)
        ws, aws, items = ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(2000, 2048)), ws_of(256), a.items()
        start = [t.clone() for t in a.tensors()]

        def run(stream, c=c, j=j, a=a, q=q, k=k, v=v, dqkv=dqkv, h=h, out=out, dx=dx, dy=dy, rq=rq, rp=rp, dgq=dgq, dgp=dgp, am=am, ws=ws,
                aws=aws, items=items):
            for _ in range(4):
                fp8.fp8_rope_qkv_fwd(c.qkv, 8, 2, *c.how, q, k, v, stream=stream)
                fp8.fp8_rope_qkv_bwd(c.dq, c.dk, c.dv, c.qkv, *c.how, dqkv, stream=stream)
                fp8.fp8_block_norm_fwd(*j.ins(), j.eps, h, out, r_post=rq, r_pre=rp, stream=stream)
                fp8.fp8_block_norm_bwd(j.dout, j.dh, h, j.y, None, j.gq, j.gp, rq, rp, *j.how, dx, dy, None, dgq, dgp, ws, amax_out=am,
                                       stream=stream)
                fp8.fp8_adamw(items, a.lr, a.step, a.b1, a.b2, a.eps, aws, norm=a.norm, max_norm=0.5, seed=7, stream=stream)

        outs.append((run, [q, k, v, dqkv, h, out, dx, dy, dgq, dgp, am], a, start))
    torch.cuda.synchronize()
    want = []
    for run, made, a, start in outs:                               # one after the other
        run(None)
        torch.cuda.synchronize()
        want.append([t.clone() for t in made + a.tensors()])
        for t, s in zip(a.tensors(), start):
            t.copy_(s)
        for t in made:
            t.fill_(2)
    torch.cuda.synchronize()
    for (run, *_), stream in zip(outs, (g1, g2)):
        run(stream)
    torch.cuda.synchronize()
    for (_, made, a, _), w in zip(outs, want):
        assert all(torch.equal(t, x) for t, x in zip(made + a.tensors(), w))


def test_joint_rows_of_zeros():
    T, D = 5, 72
    zero = torch.zeros((T, D), dtype=BF16, device="cuda")
    g = torch.ones(D, device="cuda")
    h, out = full((T, D)), full((T, D))
    fp8.fp8_block_norm_fwd(zero, zero, None, g, g, fp8.NORM_RMS, 0, 1.0, 1.0, 1e-5, h, out)
    assert (h == 0).all() and (out == 0).all()
    one = zero.clone()
    one[2] = 1.0
    fp8.fp8_block_norm_fwd(one, one, None, g, g, fp8.NORM_RMS, 0, 1.0, 1.0, 0.0, h, out)             # without eps: NaN in those rows alone
    assert torch.isnan(h[[0, 1, 3, 4]]).all() and (h[2] == 2).all() and (out[2] == 1).all()


def test_joint_beyond_32_bit_offsets():
    T, D = 140000, 16384
    x = torch.empty((T, D), dtype=BF16, device="cuda")                            # 2.3e9 elements
    assert x.numel() > 2 ** 31
    x.fill_(1.0)
    last = rnd(gen(3), 40, D, dtype=BF16)
    x[-40:] = last
    g = torch.ones(D, device="cuda")
    out, rp = torch.empty_like(x), full((T,), 0, F32)
    fp8.fp8_block_norm_fwd(x, None, None, None, g, fp8.NORM_NONE, 0, 1.0, 1.0, 1e-5, None, out, r_pre=rp)
    want, rp2 = full((40, D)), full((40,), 0, F32)
    fp8.fp8_block_norm_fwd(last, None, None, None, g, fp8.NORM_NONE, 0, 1.0, 1.0, 1e-5, None, want, r_pre=rp2)
    assert torch.equal(out[-40:], want) and torch.equal(rp[-40:], rp2) and (out[:-40] == 1).all()
    dx, dx2, dg = torch.empty_like(x), full((40, D)), full((D,), 0, F32)
    fp8.fp8_block_norm_bwd(out, None, x, None, None, None, g, None, rp, fp8.NORM_NONE, 0, 1.0, 1.0, dx, None, None, None, dg,
                           ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(T, D)))
    fp8.fp8_block_norm_bwd(want, None, last, None, None, None, g, None, rp2, fp8.NORM_NONE, 0, 1.0, 1.0, dx2, None, None, None, dg,
                           ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(40, D)))
    # the two launches split rows alike (one row at a time on a CTA): the same results
    assert torch.equal(dx[-40:], dx2)


@pytest.mark.parametrize("T,D", [(2, 64), (4, 520), (300, 1600), (20, 4096), (9, 8200), (5, 16384)])
@pytest.mark.parametrize("mode", [fp8.GATE_LINEAR, fp8.GATE_SIGMOID])
@pytest.mark.parametrize("post", [fp8.NORM_LAYERSCALE, fp8.NORM_NONE])
def test_joint_of_gates_that_are_not_finite(T, D, mode, post):
    """NaN and the two infinities in a gate, element by element: what the formula gives, both ways and in the amax; a closed sigmoid
    leaves the residual stream and gradients of exactly 0."""
    c = JointCase(T, D, post, mode, False)
    c.gate.clamp_(-60, 60)
    bad = torch.tensor([NAN, math.inf, -math.inf, -200.0], dtype=BF16)
    places = [(1, 0), (T - 1, D - 4)]
    for t, j in places:
        c.gate[t, j:j + 4] = bad
    s, slope, extra = c.weight()
    _, z = c.z()
    h, amax = full((T, D)), scalar(-1)
    fp8.fp8_block_norm_fwd(*c.ins(), c.eps, h, None, amax_out=amax)
    G = c.dh.to(F64)
    dx, dy, dg, dgq, a2 = full((T, D)), full((T, D)), full((T, D)), full((D,), 0, F32) if c.gq is not None else None, scalar(-1)
    ws = ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(T, D))
    fp8.fp8_block_norm_bwd(None, c.dh, None, c.y, c.gate, c.gq, None, None, None, *c.how, dx, dy, dg, dgq, None, ws, amax_out=a2)
    ref = c.a * c.x.to(F64) + c.b * s * z
    dgate, grad = c.b * G * z * slope, c.b * G * s * (c.gq.to(F64) if c.gq is not None else 1.0)
    sizes = (ref.abs() + 2 * (c.a * c.x.to(F64)).abs(), dgate.abs(), grad.abs())
    for got, want, size in zip((h, dg, dy), (ref, dgate, grad), sizes):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        far = torch.isinf(want)
        assert torch.equal(got[far].to(F64), want[far])
        there = torch.isfinite(want)
        more = extra if isinstance(extra, float) else extra.nan_to_num(0.0, 0.0, 0.0)[there].clamp(max=200.0)
        within(got[there], want[there], (HALF[BF16] + (64 + 2 * more) * U) * size[there] + 2.0 ** -126)
    assert math.isnan(amax.item()) and math.isnan(a2.item())
    if mode == fp8.GATE_SIGMOID:
        for t, j in places:
            assert torch.isnan(dg[t, j]) and (dg[t, j + 1:j + 4] == 0).all() and (dy[t, j + 2:j + 4] == 0).all()
            assert torch.equal(h[t, j + 2:j + 4], (c.a * c.x[t, j + 2:j + 4].float()).to(BF16))
    scale, h8, h2, d8 = scalar(37.0), full((T, D), 0xEE, U8), full((T, D)), full((T, D), 0xEE, U8)
    fp8.fp8_block_norm_fwd_q(*c.ins(), c.eps, scale, fp8.E4M3, h2, None, h8)
    fp8.fp8_block_norm_bwd_q(None, c.dh, None, c.y, c.gate, c.gq, None, None, None, *c.how, scale, fp8.E5M2, dx, None, d8, dg, dgq, None, ws)
    assert torch.equal(h8, codes_of(h, scale, fp8.E4M3)) and torch.equal(d8, codes_of(dy, scale, fp8.E5M2))


@pytest.mark.parametrize("mode", [fp8.GATE_LINEAR, fp8.GATE_SIGMOID])
def test_joint_row_of_a_broken_gate(mode):
    """Behind both norms a NaN in a gate is its whole row's, and no other's."""
    T, D = 40, 1032
    c, d = (JointCase(T, D, fp8.NORM_RMS, mode, True) for _ in range(2))
    c.gate[7, 500] = NAN
    rows = torch.arange(T, device="cuda") != 7
    made = []
    for x in (c, d):
        h, out, rq, rp, amax = full((T, D)), full((T, D)), full((T,), 0, F32), full((T,), 0, F32), scalar(-1)
        fp8.fp8_block_norm_fwd(*x.ins(), x.eps, h, out, r_post=rq, r_pre=rp, amax_out=amax)
        dx, dy, dg, dgq, dgp, a2 = full((T, D)), full((T, D)), full((T, D)), full((D,), 0, F32), full((D,), 0, F32), scalar(-1)
        fp8.fp8_block_norm_bwd(x.dout, x.dh, h, x.y, x.gate, x.gq, x.gp, rq, rp, *x.how, dx, dy, dg, dgq, dgp,
                               ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(T, D)), amax_out=a2)
        made.append((h, out, rp, dx, dy, dg, amax, a2, dgq, dgp))
    for got, want in zip(made[0][:6], made[1][:6]):
        assert torch.equal(got[rows], want[rows])
    h, out, rp, dx, dy, dg, amax, a2, dgq, dgp = made[0]
    assert torch.isnan(h[7]).sum() == 1 and torch.isnan(rp[7]) and all(torch.isnan(x[7]).all() for x in (out, dx, dy, dg))
    assert math.isnan(amax.item()) and math.isnan(a2.item()) and torch.isnan(dgq).all() and torch.isnan(dgp).all()


# ------------------------------------------------------------------------------------------------ AdamW
def mix(x):
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_bits(seed, t, item, n, start=0):
    key = mix(mix(mix(seed & 0xFFFFFFFF) ^ (seed >> 32)) ^ t)
    key = mix((key + item) & 0xFFFFFFFF)
    i = torch.arange(start, start + n, device="cuda")
    hi = i >> 32
    return mix((mix((key + hi) & 0xFFFFFFFF) + (i & 0xFFFFFFFF)) & 0xFFFFFFFF)


def blocks(x):
    pad = -x.numel() % 128
    return torch.cat([x.reshape(-1), x.new_zeros(pad)]).view(-1, 128)


def two(e):
    """2^e of whole numbers in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(F64)


def decode(codes, exps, n):
    """Values of 8-bit moments in 64 bits."""
    v = blocks(codes.reshape(-1)).view(torch.float8_e4m3fn).to(F64)
    return (v * two(exps.int()[:, None] - 127)).view(-1)[:n]


def check_codes(codes, exps, want, size, bits, floor):
    """8-bit moments against the values (64 bits; off by 32 u of `size` in the call) that they were made from: the block's exponent,
    and each value rounded away from zero exactly where its random bits say so, but for those within the call's rounding of the border."""
    n = want.numel()
    w, slack = blocks(want), 32 * U * blocks(size)
    top = w.abs().amax(1)
    # a / 448 = f 2^k with f in [1/2, 1): the power above is 2^k, or 2^(k - 1) where f is 1/2
    power = lambda v: torch.where(v > 0, (q := torch.frexp(v / 448.0)).exponent - (q.mantissa == 0.5).int(), -200).clamp(min=-126)  # noqa: E731
    e = exps.to(F64) - 127
    off = slack.amax(1)
    assert ((e == power(top)) | (e == power(top - off)) | (e == power(top + off))).all()
    unit = two(-e[:, None])
    y, slack = (w.abs() * unit).view(-1)[:n], (slack * unit).view(-1)[:n]
    octave = torch.frexp(y.clamp(min=2.0 ** -6)).exponent - 1
    step = two(octave - 3)
    part = y / step + bits.to(F64) / 65536.0
    units = torch.floor(part)
    if floor:
        units = torch.where((y > 0) & (units == 0), 1.0, units)
    value = blocks(codes.reshape(-1)).view(torch.float8_e4m3fn).to(F64).view(-1)[:n]
    away = lambda v, border: (v - border).abs() > slack + 2.0 ** -28       # FP32 next to 2^-6, where the smallest steps are cut  # noqa: E731
    sure = away(part * step, part.round() * step) & away(y, two(octave)) & away(y, two(octave + 1))
    expect = units * step * torch.sign(w).view(-1)[:n]
    assert (value[sure] == expect[sure]).all()
    assert sure.to(F64).mean() > 0.98 or n < 200
    assert ((value.abs() - y).abs() <= step * (1 + 2.0 ** -10) + slack).all()


class AdamCase:
    def __init__(self, sizes, bits, gdt, seed=0, p16=True, p8=True, zero=False):
        g = gen(sum(sizes) % 1000 + seed)
        self.sizes, self.bits = sizes, bits
        self.p = [rnd(g, n, std=0.02) for n in sizes]
        self.g = [rnd(g, n, std=1e-3 * (1 + i % 3), dtype=gdt) for i, n in enumerate(sizes)]
        for x in self.g:
            x[: x.numel() // 7] = 0                                  # rows that no token touched
        if bits == 32:
            self.m, self.v = [rnd(g, n, std=1e-4) * (not zero) for n in sizes], [rnd(g, n, std=1e-3).square() * (not zero) for n in sizes]
            self.me = self.ve = None
        else:
            pick = lambda hi: [torch.randint(0, hi, (n,), generator=g, device="cuda").to(U8) * (not zero) for n in sizes]  # noqa: E731
            ex = lambda lo: [torch.randint(lo, lo + 6, (-(-n // 128),), generator=g, device="cuda").to(U8) * (not zero) for n in sizes]  # noqa: E731
            self.m = [torch.where(x == 127, 1, torch.where(x == 255, 0x81, x.int())).to(U8) for x in pick(256)]
            self.v = pick(127)
            self.me, self.ve = ex(104), ex(106)
        self.p16 = [full((n,)) for n in sizes] if p16 else None
        self.p8 = [full((n,), 0xEE, U8) for n in sizes] if p8 else None
        self.q = torch.rand(len(sizes), generator=g, device="cuda") * 500 + 100
        self.amax = full((len(sizes),), -1.0, F32)
        self.decay = [0.1 * (i % 3) for i in range(len(sizes))]
        self.lr, self.step, self.norm = scalar(3e-4), torch.full((1,), 4, dtype=torch.int32, device="cuda"), scalar(2.0)
        self.b1, self.b2, self.eps, self.seed = 0.9, 0.999, 1e-8, 0xDEADBEEF12345678

    def items(self):
        return fp8.fp8_adamw_items(self.p, self.g, self.m, self.v, self.decay, m_exps=self.me, v_exps=self.ve, params16=self.p16,
                                   params8=self.p8, q_scales=self.q, amaxes=self.amax, fmt=fp8.E4M3)

    def call(self, items, **more):
        ws = ws_of(fp8.fp8_adamw_workspace_bytes(items))
        fp8.fp8_adamw(items, self.lr, self.step, self.b1, self.b2, self.eps, ws, norm=self.norm, max_norm=0.5, seed=self.seed, **more)

    def tensors(self):
        return [t for x in (self.p, self.m, self.v, self.me, self.ve, self.p16, self.p8, [self.amax, self.step]) if x is not None for t in x]

    def moments(self, i):
        if self.bits == 32:
            return self.m[i].to(F64), self.v[i].to(F64)
        n = self.sizes[i]
        return decode(self.m[i], self.me[i], n), decode(self.v[i], self.ve[i], n).square()


@pytest.mark.parametrize("sizes", [[1], [7], [8], [127], [128], [129], [4096], [4097, 1, 15], [2048 * 3 + 8, 5000, 3, 128 * 9 + 1],
                                   [100003], [33] * 300, [1, 2, 3] * 200 + [70000]])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt", [BF16, F32])
def test_adamw(sizes, bits, gdt):
    c = AdamCase(sizes, bits, gdt)
    before = [(*c.moments(i), c.p[i].to(F64)) for i in range(len(sizes))]
    c.call(c.items())
    t = 5
    assert c.step.item() == t
    factor = 0.5 / (2.0 + 1e-6)
    lr = float(np.float32(3e-4))
    for i, n in enumerate(sizes):
        if i > 8 and i % 37:
            continue
        m0, v0, p0 = before[i]
        g = c.g[i].to(F64) * factor
        # each term is off by a few u of itself: the factor, the rates' FP32 values, the products, the sum
        m, m_mag = c.b1 * m0 + (1 - c.b1) * g, c.b1 * m0.abs() + (1 - c.b1) * g.abs()
        v = c.b2 * v0 + (1 - c.b2) * g * g
        root = (v / (1 - c.b2 ** t)).sqrt()
        rate = lr / (1 - c.b1 ** t)
        wd = float(np.float32(c.decay[i]))
        p = p0 * (1 - lr * wd) - rate * m / (root + c.eps)
        within(c.p[i], p, 4 * U * p0.abs() + 32 * U * rate * m_mag / (root + c.eps) + U * p.abs())
        if bits == 32:
            within(c.m[i], m, 8 * U * m_mag)
            within(c.v[i], v, 8 * U * v)
        else:
            r = random_bits(c.seed, t, i, n)
            check_codes(c.m[i], c.me[i], m, m_mag, r & 0xFFFF, False)
            check_codes(c.v[i], c.ve[i], v.sqrt(), v.sqrt(), r >> 16, True)
        assert torch.equal(c.p16[i], c.p[i].to(BF16)) and c.amax[i].item() == amax_of(c.p16[i])
        assert torch.equal(c.p8[i], codes_of(c.p16[i], c.q[i:i + 1], fp8.E4M3))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_passes_over_empty_tensors(bits):
    """Their place in the list still counts: it is part of the random bits' key."""
    c, d = AdamCase([300, 0, 5000, 0], bits, F32, seed=3), AdamCase([300, 0, 5000, 0], bits, F32, seed=3)
    c.amax.fill_(5.0)
    c.call(c.items())
    d.call(d.items())
    assert c.step.item() == 5 and c.amax[1].item() == 5.0 and c.amax[3].item() == 5.0
    assert all(torch.equal(x, y) for x, y in zip(c.p + c.m + c.v, d.p + d.m + d.v))
    if bits == 8:
        e = AdamCase([300, 0, 5000, 0], bits, F32, seed=3)
        m, v = e.moments(2)
        e.call(e.items())
        g = e.g[2].to(F64) * (0.5 / (2.0 + 1e-6))
        new, size = e.b1 * m + (1 - e.b1) * g, e.b1 * m.abs() + (1 - e.b1) * g.abs()
        check_codes(e.m[2], e.me[2], new, size, random_bits(e.seed, 5, 2, 5000) & 0xFFFF, False)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_zero_states_and_without_extras(bits):
    c = AdamCase([1000, 130], bits, F32, p16=False, p8=False, zero=True)
    c.norm = None
    c.step.zero_()
    p0 = [p.clone() for p in c.p]
    items = fp8.fp8_adamw_items(c.p, c.g, c.m, c.v, [0.0, 0.0], m_exps=c.me, v_exps=c.ve)
    c.call(items)
    for p, q, g in zip(c.p, p0, c.g):                              # the first step: a step of lr against the gradient's sign
        g = g.to(F64)
        want = q.to(F64) - float(np.float32(3e-4)) * g / (g.abs() + c.eps)
        within(p, want, 8 * U * q.to(F64).abs() + 64 * U * 3e-4)
        assert torch.equal(p[g == 0], q[g == 0])
    for m, v in zip(c.m, c.v):
        assert (m[:10] == 0).all() and (v[:10] == 0).all()         # untouched rows keep moments of zero


@pytest.mark.parametrize("bad", [math.inf, NAN])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_skips_a_step_whose_norm_is_not_finite(bad, bits):
    c = AdamCase([5000, 77], bits, BF16)
    c.g[0][3] = bad
    c.norm = scalar(bad)
    old = [t.clone() for t in c.tensors()]
    items = c.items()
    c.call(items)
    assert all(torch.equal(a.view(U8) if a.dtype != U8 else a, b.view(U8) if b.dtype != U8 else b) for a, b in zip(old, c.tensors()))
    c.g[0][3] = 0.0
    c.norm = scalar(0.1)                                           # below max_norm: not scaled
    c.call(items)
    assert c.step.item() == 5 and not torch.isnan(c.p[0]).any()


@pytest.mark.parametrize("bad", [math.inf, NAN, 1e30])
def test_adamw_of_gradients_that_are_not_finite_without_a_norm(bad):
    """A value that is not finite spoils its own element, not the block's others; squares that overflow likewise."""
    c, d = AdamCase([400], 8, F32), AdamCase([400], 8, F32)
    for x in (c, d):
        x.norm = None
    c.g[0][200] = bad
    d.g[0][200] = 0.0
    c.call(c.items())
    d.call(d.items())
    other = torch.arange(400, device="cuda") != 200
    assert torch.equal(c.p[0][other], d.p[0][other])
    far = (torch.arange(400, device="cuda") // 128) != 1
    assert torch.equal(c.m[0][far], d.m[0][far]) and torch.equal(c.v[0][far], d.v[0][far])
    r = decode(c.v[0], c.ve[0], 400)
    assert torch.isnan(r[200]) and not torch.isnan(r[other]).any()                  # 0.001 * 1e60 is over FP32's range
    m = decode(c.m[0], c.me[0], 400)
    assert not torch.isnan(m[other]).any() and (torch.isnan(m[200]) if bad != 1e30 else m[200] > 1e28)


@pytest.mark.parametrize("scale", [1e-20, 1e-12, 1e3, 1e12])
def test_adamw_8_bit_moments_over_the_range_of_scales(scale):
    """Blocks far from the usual size: small ones down to where squares vanish (below FP32's normal numbers: 0), large ones up to
    where they overflow."""
    c = AdamCase([1000], 8, F32)
    c.norm = None
    c.m[0].zero_(), c.v[0].zero_(), c.me[0].zero_(), c.ve[0].zero_()
    c.g[0].mul_(1e3 * scale)
    g = c.g[0].to(F64)
    c.call(c.items())
    new_m = (1 - c.b1) * g
    v = (1 - c.b2) * g * g
    gone = v < 2.0 ** -125
    check_codes(c.m[0], c.me[0], new_m, new_m.abs(), random_bits(c.seed, 5, 0, 1000) & 0xFFFF, False)
    got = decode(c.v[0], c.ve[0], 1000)
    assert (got[v < 2.0 ** -127] == 0).all()
    if not gone.any() or scale > 1e-15:
        check_codes(c.v[0], c.ve[0], v.sqrt(), v.sqrt(), random_bits(c.seed, 5, 0, 1000) >> 16, True)


@pytest.mark.parametrize("bad", [1e30, -3e38])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_squares_that_overflow(bad, bits):
    """A finite gradient whose square is over FP32's range: an infinite second moment moves nothing, in this step and in the next
    ones, whatever the moments' width; the weight only decays."""
    c = AdamCase([8, 700], bits, F32)
    c.norm = None
    c.g[1][200] = bad
    p0 = c.p[1].to(F64)
    items = c.items()
    decay = 1.0 - float(np.float32(3e-4)) * float(np.float32(c.decay[1]))
    for step in range(1, 4):
        c.call(items)
        assert abs(c.p[1][200].item() - p0[200].item() * decay ** step) <= 4 * step * U * abs(p0[200].item())
        assert all(torch.isfinite(x).all() for x in c.p)
        assert torch.equal(c.p16[1], c.p[1].to(BF16)) and c.amax[1].item() == amax_of(c.p16[1])
        assert torch.equal(c.p8[1], codes_of(c.p16[1], c.q[1:2], fp8.E4M3))
        c.g[1][200] = 1e-3
    if bits == 32:
        assert c.v[1][200].item() == math.inf


def test_adamw_8_bit_moments_next_to_the_smallest_numbers():
    """Terms and sums below FP32's normal numbers (2^-126) count as 0 with moments of 8 bits, beside an old moment above them too.
    The roots' values are FP32's next to the formula's: codes are compared away from the rounding's borders."""
    n = 1280
    c = AdamCase([n], 8, F32)
    c.norm = None
    tiny = 2.0 ** -126
    c.v[0].fill_(0x3A), c.ve[0].fill_(64)                          # roots of 1.25 * 2^-63
    c.m[0].fill_(0x38), c.me[0].fill_(6)                           # 2^-121
    v_old, m_old = 1.5625 * tiny, 32.0 * tiny
    small = torch.arange(n, device="cuda") % 2 == 0                # every other new term lies below the normal numbers
    c.g[0].copy_(torch.where(small, math.sqrt(0.5 * tiny / 0.001), math.sqrt(4.0 * tiny / 0.001)))
    g = c.g[0].to(F64)
    c.call(c.items())
    terms = (1 - c.b2) * g * g
    v = c.b2 * v_old + torch.where(terms < tiny, 0.0, terms)
    assert torch.equal(terms < tiny, small)
    r = random_bits(c.seed, 5, 0, n)
    check_codes(c.v[0], c.ve[0], v.sqrt(), v.sqrt(), r >> 16, True)
    m = c.b1 * m_old + (1 - c.b1) * g
    check_codes(c.m[0], c.me[0], m, m.abs(), r & 0xFFFF, False)
    # first moments: new terms of half the smallest normal number beside an old one above it, and alone
    c = AdamCase([n], 8, F32)
    c.norm = None
    c.v[0].fill_(0x38), c.ve[0].fill_(120)
    c.m[0].copy_(torch.where(small, 0x40, 0).to(U8)), c.me[0].fill_(1)
    c.g[0].fill_(5.0 * tiny)                                       # a tenth of it is tiny / 2
    c.call(c.items())
    got = decode(c.m[0], c.me[0], n)
    kept = 0.9 * 2.0 * tiny
    r = random_bits(c.seed, 5, 0, n)
    assert (got[~small] == 0).all()
    check_codes(c.m[0], c.me[0], torch.where(small, kept, 0.0).to(F64), torch.where(small, kept, 0.0).to(F64), r & 0xFFFF, False)


def test_adamw_random_rounding_is_unbiased_and_repeats():
    """Small changes of a large second moment: rounded to nearest they would be lost.  2^20 values between two codes: the mean
    of the stored values is within 5 deviations (step / 2 / 2^10 each) of the value, the two codes are the neighbours."""
    n = 1 << 20
    one = lambda: AdamCase([n], 8, F32)  # noqa: E731
    c = one()
    c.m[0].fill_(0x38)                                             # 1.0
    c.me[0].fill_(120)
    c.v[0].fill_(0x3C)                                             # 1.5
    c.ve[0].fill_(118)
    for t in (c.m[0], c.v[0]):
        t[::128] = 0x7E                                            # 448 keeps the blocks' scales
    c.g[0].zero_()
    c.b1, c.b2 = 0.97, 0.98
    c.call(c.items())
    body = torch.arange(n, device="cuda") % 128 != 0
    for codes, exps, was, e, new in ((c.m[0], c.me[0], 1.0, 120, 0.97), (c.v[0], c.ve[0], 1.5, 118, 1.5 * math.sqrt(0.98))):
        value = decode(codes, exps, n)[body] * 2.0 ** (127 - e)
        step = 0.0625 if new < 1 else 0.125
        assert set(value.unique().tolist()) <= {math.floor(new / step) * step, math.ceil(new / step) * step}
        assert abs(value.mean().item() - new) <= 5 * step / 2 / 2 ** 10
    again, other = one(), one()
    for k, x in enumerate((again, other)):
        x.call(x.items())
    assert all(torch.equal(a, b) for a, b in zip(again.tensors(), other.tensors()))
    third = one()
    third.seed += 1
    third.call(third.items())
    assert torch.equal(third.p[0], again.p[0]) and not torch.equal(third.m[0], again.m[0])


def test_adamw_beyond_32_bit_offsets():
    n, k = (1 << 32) + 5000, 6000
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    m, v = torch.zeros(n, dtype=U8, device="cuda"), torch.zeros(n, dtype=U8, device="cuda")
    me, ve = torch.zeros(-(-n // 128), dtype=U8, device="cuda"), torch.zeros(-(-n // 128), dtype=U8, device="cuda")
    g[-k:] = rnd(gen(4), k, std=1e-3, dtype=BF16)
    lr, step = scalar(1e-3), torch.zeros(1, dtype=torch.int32, device="cuda")
    items = fp8.fp8_adamw_items([p], [g], [m], [v], [0.0], m_exps=[me], v_exps=[ve])
    fp8.fp8_adamw(items, lr, step, 0.9, 0.95, 1e-8, ws_of(256), seed=99)
    d = g[-k:].to(F64)
    want = -float(np.float32(1e-3)) * d / (d.abs() + 1e-8)
    within(p[-k:], want, 64 * U * 1e-3 * torch.ones_like(want))
    assert p[:-k].count_nonzero() == 0 and m[:-k].count_nonzero() == 0
    start = n - k
    lead = start % 128                                             # the first whole block
    first = start + (128 - lead) % 128
    r = random_bits(99, 1, 0, n - first, first)
    tail = slice(first, n)
    new_m, new_r = 0.1 * g[tail].to(F64), math.sqrt(0.05) * g[tail].to(F64).abs()
    check_codes(m[tail], me[first // 128:], new_m, new_m.abs(), r & 0xFFFF, False)
    check_codes(v[tail], ve[first // 128:], new_r, new_r, r >> 16, True)


# ------------------------------------------------------------------------------------------------ streams, graphs, together
def test_calls_in_a_graph_and_on_other_streams_give_the_same():
    c = RopeCase(70, 8, 2, 128, 64, fp8.QK_RMS, True, torch.int64)
    j = JointCase(300, 1600, fp8.NORM_RMS, fp8.GATE_SIGMOID, True)
    a = AdamCase([5000, 33, 128], 8, BF16)
    items, ws, aws = a.items(), ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(300, 1600)), ws_of(256)
    q, k, v, dqkv, ramax = full((70, 8, 128)), full((70, 2, 128)), full((70, 2, 128)), full((70, c.W)), full((3,), 0, F32)
    h, out, rq, rp, amax = full((300, 1600)), full((300, 1600)), full((300,), 0, F32), full((300,), 0, F32), scalar(0)
    dx, dy, dg, dgq, dgp = full((300, 1600)), full((300, 1600)), full((300, 1600)), full((1600,), 0, F32), full((1600,), 0, F32)

    def calls():
        fp8.fp8_rope_qkv_fwd(c.qkv, 8, 2, *c.how, q, k, v, amax_out=ramax)
        fp8.fp8_rope_qkv_bwd(c.dq, c.dk, c.dv, c.qkv, *c.how, dqkv)
        fp8.fp8_block_norm_fwd(*j.ins(), j.eps, h, out, r_post=rq, r_pre=rp, amax_out=amax)
        fp8.fp8_block_norm_bwd(j.dout, j.dh, h, j.y, j.gate, j.gq, j.gp, rq, rp, *j.how, dx, dy, dg, dgq, dgp, ws)
        fp8.fp8_adamw(items, a.lr, a.step, a.b1, a.b2, a.eps, aws, norm=a.norm, max_norm=0.5, seed=3)

    outs = [q, k, v, dqkv, ramax, h, out, rq, rp, amax, dx, dy, dg, dgq, dgp]
    state = [t.clone() for t in a.tensors()]

    def reset():
        for t, s in zip(a.tensors(), state):
            t.copy_(s)
        for t in outs:
            t.fill_(3)

    calls()
    calls()
    want = [t.clone() for t in outs + a.tensors()]
    side = torch.cuda.Stream()
    reset()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
        calls()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, w) for t, w in zip(outs + a.tensors(), want))
    reset()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls()
    reset()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(outs + a.tensors(), want))


def test_python_refuses_before_any_call():
    c = RopeCase(6, 2, 1, 32, 32, fp8.QK_NONE, False, None)
    q, k, v = full((6, 2, 32)), full((6, 1, 32)), full((6, 1, 32))
    with pytest.raises(ValueError):
        fp8.fp8_rope_qkv_fwd(c.qkv.float(), 2, 1, *c.how, q, k, v)
    with pytest.raises(ValueError):
        fp8.fp8_rope_qkv_fwd(c.qkv.t().contiguous().t(), 2, 1, *c.how, q, k, v)          # columns strided
    with pytest.raises(ValueError):
        fp8.fp8_rope_qkv_fwd(c.qkv, 3, 1, *c.how, q, k, v)
    with pytest.raises(ValueError):
        fp8.fp8_rope_qkv_fwd(c.qkv, 2, 1, *c.how, q[:, :1], k, v)
    with pytest.raises(ValueError):
        fp8.fp8_rope_qkv_fwd(c.qkv, 2, 1, *c.how[:5], torch.zeros(5, dtype=torch.int64, device="cuda"), False, q, k, v)
    with pytest.raises(fp8.Fp8Error):
        fp8.fp8_rope_qkv_fwd(c.qkv, 2, 1, *c.how, None, None, None)
    p, g, z = torch.zeros(200, device="cuda"), torch.zeros(200, device="cuda"), torch.zeros(200, device="cuda")
    with pytest.raises(ValueError):
        fp8.fp8_adamw_items([p, p], [g, g], [z, z.clone()], [z.clone(), z.clone()], [0.0, 0.0])         # tied weights
    with pytest.raises(ValueError):
        fp8.fp8_adamw_items([p], [g], [z.to(U8)], [z.to(U8)], [0.0])                                     # no exponents
    with pytest.raises(ValueError):
        fp8.fp8_adamw_items([p], [g], [z], [torch.zeros(100, device="cuda")], [0.0])
    with pytest.raises(ValueError):
        fp8.fp8_adamw_items([p], [g], [z], [z.clone()], [0.0], params8=[z.to(U8)])


def test_a_block_trains_through_the_calls():
    """The attention half of a block and the optimizer as they are used: norm in front, QKV projection, rotation, attention, output
    projection, joint with the norm behind and in front of what comes next; back; clip and AdamW that leaves the next step's FP8
    weights.  Every new call is held against 64 bits on the inputs that it got; the whole gradient of the weights lies along
    that of the same half block without FP8 (operands of 3 and 2 bits: E4M3 is off by 2^-4 of a value at most, E5M2 by 2^-3, so
    products of them by 0.2 in norm, over four products in a row by less than 0.5: a cosine above 0.85)."""
    T, Hq, Hkv, d = 256, 4, 2, 64
    D, W = Hq * d, (Hq + 2 * Hkv) * d
    g = gen(77)
    x = rnd(g, T, D, dtype=BF16)
    wq, wo = rnd(g, W, D, std=D ** -0.5), rnd(g, D, D, std=D ** -0.5)
    gp1, gq, gp2 = (1 + rnd(g, D, std=0.1) for _ in range(3))
    cos, sin = full((T, d // 2), 0, F32), full((T, d // 2), 0, F32)
    fp8.fp8_rope_table(cos, sin, 10000.0)
    e8 = lambda *s: torch.empty(s, dtype=U8, device="cuda")  # noqa: E731
    eb = lambda *s: torch.empty(s, dtype=BF16, device="cuda")  # noqa: E731
    ef = lambda *s: torch.empty(s, dtype=F32, device="cuda")  # noqa: E731

    def quantized(t, fmt):
        t = t.to(BF16)
        out, a, s, si = e8(*t.shape), ef(1), ef(1), ef(1)
        fp8.fp8_quantize(t, fmt, out, None, a, s, si)
        return out, si

    how = (fp8.QK_RMS, 0.0, 1e-6, cos, sin, None, False)
    wq8, wqi = quantized(wq, fp8.E4M3)
    wo8, woi = quantized(wo, fp8.E4M3)
    s_in, s_in_inv = scalar(64.0), scalar(1 / 64.0)
    h8, rp1 = e8(T, D), ef(T)
    fp8.fp8_block_norm_fwd_q(x, None, None, None, gp1, fp8.NORM_NONE, 0, 1.0, 1.0, 1e-5, s_in, fp8.E4M3, None, None, h8, r_pre=rp1)
    qkv = eb(T, W)
    fp8.fp8_linear_fwd(h8, wq8, s_in_inv, wqi, qkv)
    sc, sc_inv = torch.tensor([64.0, 64.0, 64.0], device="cuda"), scalar(1 / 64.0)
    q8, k8, v8, amax = e8(1, T, Hq, d), e8(1, T, Hkv, d), e8(1, T, Hkv, d), ef(3)
    fp8.fp8_rope_qkv_fwd_q(qkv, Hq, Hkv, *how, sc, fp8.E4M3, q8[0], k8[0], v8[0], amax_out=amax)
    assert (amax * sc < 448).all()
    o, lse = eb(1, T, Hq, d), ef(1, Hq, T)
    fp8.fp8_attention_fwd(q8, k8, v8, sc_inv, sc_inv, sc_inv, d ** -0.5, True, o, lse, None)
    o8, oi = quantized(o.view(T, D), fp8.E4M3)
    y, h, out, rq, rp2 = eb(T, D), eb(T, D), eb(T, D), ef(T), ef(T)
    fp8.fp8_linear_fwd(o8, wo8, oi, woi, y)
    fp8.fp8_block_norm_fwd(x, y, None, gq, gp2, fp8.NORM_RMS, 0, 1.0, 0.5, 1e-5, h, out, r_post=rq, r_pre=rp2)
    # back
    dout, dh = rnd(g, T, D, std=1e-3, dtype=BF16), rnd(g, T, D, std=1e-3, dtype=BF16)
    dx, dy, dy8, sy, syi = eb(T, D), eb(T, D), e8(T, D), scalar(2.0 ** 20), scalar(2.0 ** -20)
    dgq, dgp2, dgp1 = ef(D), ef(D), ef(D)
    ws = ws_of(fp8.fp8_block_norm_bwd_workspace_bytes(T, D))
    fp8.fp8_block_norm_bwd_q(dout, dh, h, y, None, gq, gp2, rq, rp2, fp8.NORM_RMS, 0, 1.0, 0.5, sy, fp8.E5M2, dx, dy, dy8, None, dgq, dgp2, ws)
    do, dwo, dwq = eb(1, T, Hq, d), ef(D, D), ef(W, D)
    fp8.fp8_linear_dgrad_rm(dy8, wo8, syi, woi, do.view(T, D))
    fp8.fp8_linear_wgrad_rm(dy8, o8, syi, oi, dwo)
    do8, doi = quantized(do.view(T, D), fp8.E5M2)
    dq, dk, dv = eb(1, T, Hq, d), eb(1, T, Hkv, d), eb(1, T, Hkv, d)
    aws = torch.empty(fp8.fp8_attention_workspace_bytes(1, 1, T, Hq, Hkv, d), dtype=U8, device="cuda")
    fp8.fp8_attention_bwd(q8, k8, v8, do8.view(1, T, Hq, d), o, lse, sc_inv, sc_inv, sc_inv, doi, d ** -0.5, scalar(2.0 ** 22), True, dq, dk, dv, aws)
    dqkv, dqkv8, samax = eb(T, W), e8(T, W), ef(1)
    fp8.fp8_rope_qkv_bwd_q(dq[0], dk[0], dv[0], qkv, *how, sy, fp8.E5M2, dqkv8, dqkv, samax)
    dn = eb(T, D)
    fp8.fp8_linear_dgrad_rm(dqkv8, wq8, syi, wqi, dn)
    fp8.fp8_linear_wgrad_rm(dqkv8, h8, syi, s_in_inv, dwq)
    dx0 = eb(T, D)
    fp8.fp8_block_norm_bwd(dn, dx, x, None, None, None, gp1, None, rp1, fp8.NORM_NONE, 0, 1.0, 1.0, dx0, None, None, None, dgp1, ws)
    # each new call on what it got
    c = RopeCase(T, Hq, Hkv, d, d, fp8.QK_RMS, False, None, N=T)
    c.qkv, c.cos, c.sin, c.dq, c.dk, c.dv, c.eps = qkv, cos, sin, dq[0], dk[0], dv[0], 1e-6
    ref, size = (t.reshape(T, -1) for t in c.backward())
    within(dqkv, ref, HALF[BF16] * ref.abs() + 64 * U * size)
    # the same half block in 64 bits
    leaves = [t.to(F64).requires_grad_() for t in (x, wq, wo, gp1, gq, gp2)]
    X, WQ, WO, A, B, C = leaves
    rms = lambda t, e: t * (t.square().mean(-1, keepdim=True) + e).rsqrt()  # noqa: E731
    u = (rms(X, 1e-5) * A) @ WQ.t()
    qk, vv = u.view(T, -1, d).split([Hq + Hkv, Hkv], 1)
    qk = rms(qk, 1e-6)
    i, j2 = qk[..., :d // 2], qk[..., d // 2:]
    cc, ss = cos.to(F64)[:, None], sin.to(F64)[:, None]
    qk = torch.cat([i * cc - j2 * ss, j2 * cc + i * ss], -1)
    Q, K = qk.split([Hq, Hkv], 1)
    K, V = K.repeat_interleave(Hq // Hkv, 1), vv.repeat_interleave(Hq // Hkv, 1)
    S = torch.einsum("thd,shd->hts", Q, K) * d ** -0.5
    S = S.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), -math.inf)
    Y = torch.einsum("hts,shd->thd", S.softmax(-1), V).reshape(T, D) @ WO.t()
    Hh = X + 0.5 * rms(Y, 1e-5) * B
    loss = (Hh * dh.to(F64)).sum() + (rms(Hh, 1e-5) * C * dout.to(F64)).sum()
    want = torch.autograd.grad(loss, leaves)
    for got, ref in zip((dx0, dwq, dwo, dgp1, dgq, dgp2), want):
        got = got.to(F64)
        assert ((got * ref).sum() / (got.norm() * ref.norm())).item() > 0.85
    # clip, step, and the FP8 weights that the next step's products read
    params, grads = [wq, wo, gp1, gq, gp2], [dwq, dwo, dgp1, dgq, dgp2]
    eight = [True, True, False, False, False]
    ms = [torch.zeros_like(p, dtype=U8 if b else F32) for p, b in zip(params, eight)]
    vs = [torch.zeros_like(p, dtype=U8 if b else F32) for p, b in zip(params, eight)]
    exps = lambda: [torch.zeros(-(-p.numel() // 128), dtype=U8, device="cuda") for p in params]  # noqa: E731
    p8 = [wq8, wo8, None, None, None]
    scales, amaxes = torch.full((5,), 1024.0, device="cuda"), ef(5)
    items = fp8.fp8_adamw_items(params, grads, ms, vs, [0.1, 0.1, 0.0, 0.0, 0.0], m_exps=exps(), v_exps=exps(), params8=p8,
                                q_scales=scales, amaxes=amaxes)
    clip = fp8.fp8_grad_items(grads)
    norm, step = ef(1), torch.zeros(1, dtype=torch.int32, device="cuda")
    old = [p.clone() for p in params]
    fp8.fp8_grad_norm(clip, norm, ws_of(fp8.fp8_grad_norm_workspace_bytes(clip)))
    fp8.fp8_adamw(items, scalar(1e-3), step, 0.9, 0.95, 1e-8, ws_of(fp8.fp8_adamw_workspace_bytes(items)), norm=norm, max_norm=1.0, seed=1)
    factor = min(1.0, 1.0 / (norm.item() + 1e-6))
    for p, q, gr, wd, a in zip(params, old, grads, (0.1, 0.1, 0, 0, 0), amaxes):
        gd = gr.to(F64) * factor
        lr = float(np.float32(1e-3))
        ref = q.to(F64) * (1 - lr * float(np.float32(wd))) - lr * gd / (gd.abs() + 1e-8)
        within(p, ref, 8 * U * q.to(F64).abs() + 64 * U * 1e-3)
        assert a.item() == amax_of(p.to(BF16))
    assert torch.equal(wq8, codes_of(wq.to(BF16), scales[:1], fp8.E4M3))
    fp8.fp8_linear_fwd(h8, wq8, s_in_inv, scalar(1 / 1024.0), qkv)               # the next step's product reads them
    torch.cuda.synchronize()
    assert fp8.fp8_device_status() == 0 and torch.isfinite(qkv.float()).all()
