"""corr_attention and its gradient where scores lie far from zero: up to the largest that their types make, near each other and far apart, in tiles
and shares that see them in any order.  What is expected is exact or bounded here; U and EPS are rows_reference's.

A score is an fp32 sum; the inputs below make sums of few powers of two, which fp32 holds, so that scores are exact.  Then
    one key above all others by more than 104 (fp32's smallest number): its weight is all of the sum and out is its v, lse its score (times scale, rounded).
        Where |score| log2 e passes 2^16 the weight is one and out is v bit by bit; below, it is a power of two's neighbour that may be rounded: U and 16 EPS.
    n keys of one score: out is their mean: weights, rounded as operands, are the same for all, and the sums' (4 Lk + 16) EPS.
    scores S + t with t small: weights e^(t - max t) with (8 (|t - max t| + 1) + 6 (Lk / 16 + 1)) EPS, as of scores near zero.
The gradient reads lse, which fp32 holds to EPS |lse|: a weight is off by that, relative, besides.  One key above all others has a weight of one, the others zero.
"""
import pytest

import maps_reference as ref
from rows_reference import EPS, U, rounded

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)
#: rows of a call: one wave and shares of the keys, weights in two parts, one block a wave, two blocks
ROWS = (1, 40, 700, 2500)


def _b():
    from paper_2505_16942_amd import binding
    return binding


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return lambda *shape, sigma=1.0, dtype=F32: (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()


def _keys(scores, D, dtype, by):
    """q = (by, 1, 0, ...), k = (high, low, 0, ...) with by high + low = the scores, high a multiple of 2^-3 of the largest's exponent"""
    q = torch.zeros(D, dtype=torch.float64)
    q[0], q[1] = by, 1.0
    k = torch.zeros(len(scores), D, dtype=torch.float64)
    k[:, 0] = scores / by
    low = scores - k[:, 0].to(dtype).double() * by
    k[:, 0], k[:, 1] = k[:, 0].to(dtype).double(), low
    assert torch.equal(k.to(dtype).double(), k) and torch.equal(k @ q, scores) and torch.equal(scores.float().double(), scores)
    return q.to(dtype).cuda(), k.to(dtype).cuda()


def _run(q, k, v, g, scale):
    b = _b()
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), float("nan"), device="cuda")
    out = b.corr_attention(q, k, v, scale=scale, lse=lse)
    return out, lse, b.corr_attention_backward(q, k, v, out, lse, g, scale=scale)


def _is_value(what, out, v, score):
    if abs(score) * 1.44 > 65540:
        assert torch.equal(out, v.expand_as(out)), what
    else:
        v = v.double().cpu().expand(out.shape)
        ref.check(what, out, v, ((0.0 if out.dtype == F32 else U[out.dtype]) + 16 * EPS) * v.abs() + rounded(v, out.dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Lq", ROWS)
@pytest.mark.parametrize("D", [24, 64, 128, 256])
def test_one_key_above_all(D, Lq, dtype):
    """From scores of a few hundred to the largest, of either sign (all others lower), the one at each end and in between."""
    new = _gen(D + Lq)
    Lk = 300
    v, g = new(1, Lk, 1, D, dtype=dtype), new(1, Lq, 1, D, dtype=dtype)
    big = (2.0 ** 15, 2.0 ** 15) if dtype == F16 else (2.0 ** 58, 2.0 ** 60)
    for x, y in ((16.0, 1.5), (64.0, 64.0), (1708.0, 1708.0), (1024.0, 8192.0), big):
        x, y = (torch.tensor(t).to(dtype).item() for t in (x, y))
        for place in (0, 131, Lk - 1):
            for sign in (1.0, -1.0):
                q = torch.full((1, Lq, 1, D), x, dtype=dtype, device="cuda")
                k = torch.zeros(1, Lk, 1, D, dtype=dtype, device="cuda") if sign > 0 else torch.full((1, Lk, 1, D), -1.5 * y, dtype=dtype, device="cuda")
                if sign < 0 and not k.isfinite().all():
                    continue
                k[0, place] = sign * y
                score = sign * D * x * y
                what = "%s %g x %g at %d" % (dtype, x, sign * y, place)
                for scale in (1.0, D ** -0.5):
                    if abs(score) * scale < 257:
                        continue
                    out, lse, (dq, dk, dv) = _run(q, k, v, g, scale)
                    _is_value(what, out, v[:, place:place + 1], score * scale)
                    exact = torch.tensor(score, dtype=torch.float64) * torch.tensor(scale, dtype=F32).double()
                    assert ((lse.double().cpu() - exact).abs() <= (2 * D + 12) * EPS * exact.abs()).all(), what
                    # d_v: the sum of d_out over rows, other keys' zero; dS is what dP and delta were rounded by
                    gd = g.double().cpu()[0, :, 0]
                    ref.check(what + " d_v", dv[:, place, 0], gd.sum(0)[None], (2 * Lq + 16) * EPS * gd.abs().sum(0)[None] + rounded(gd.sum(0)[None], dtype))
                    rest = torch.arange(Lk) != place
                    assert not dv[0, rest].any() and not dk[0, rest].any(), what
                    ds = (4 * D + 16) * EPS * (gd.abs() @ v[0, place, 0].double().cpu().abs())
                    ends = 65504.0 if dtype == F16 else 1e38
                    for name, got, most in (("d_q", dq[0, :, 0], scale * ds * abs(y)), ("d_k", dk[0, place:place + 1, 0], scale * ds.sum() * x)):
                        if most.max() < ends:
                            assert (got.double().cpu().abs() <= most.reshape(-1, 1) * 1.1 + ref.TINY[dtype]).all(), (what, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Lq", ROWS)
def test_equal_scores(Lq, dtype):
    """Every seventh key has the one far score: the mean of their values."""
    new = _gen(Lq)
    Lk, D = 400, 64
    v, g = new(1, Lk, 1, D, dtype=dtype), new(1, Lq, 1, D, dtype=dtype)
    some = torch.arange(Lk) % 7 == 3
    want = v[0, some, 0].double().cpu().mean(0)
    size = v[0, some, 0].double().cpu().abs().mean(0)
    e = (U[dtype] * (dtype != F32) + (4 * Lk + 16) * EPS) * size + rounded(want, dtype)
    for x in (1024.0, 2.0 ** 15):
        q = torch.full((1, Lq, 1, D), x, dtype=dtype, device="cuda")
        k = torch.zeros(1, Lk, 1, D, dtype=dtype, device="cuda")
        k[0, some] = x
        out, lse, _ = _run(q, k, v, g, 0.125)
        ref.check("%g" % x, out[0, :, 0], want.expand(Lq, D), e.expand(Lq, D))
        exact = x * x * 8 + some.sum().double().log()
        assert ((lse.double().cpu() - exact).abs() <= 2 * EPS * exact).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Lq", ROWS)
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_that_grow_and_fall(sign, order, Lq, dtype):
    """Scores a thousand apart, from near zero to far: every key is far above those before it, or far below, and shares of the keys end on both sides."""
    new = _gen(Lq + 5)
    Lk, D = 1000, 40
    v, g = new(1, Lk, 1, D, dtype=dtype), new(1, Lq, 1, D, dtype=dtype)
    n = torch.arange(Lk, dtype=torch.float64)
    at = {"up": n, "down": n.flip(0), "mixed": (n * 617) % Lk}[order]
    # multiples of 1024 with eight digits in two parts
    scores = 1024 * sign * (at + (sign < 0))
    q, k = _keys(scores / 8, D, dtype, 128.0)
    top = int(scores.argmax())
    q = q.expand(1, Lq, 1, D).contiguous()
    k = k.view(1, Lk, 1, D)
    out, lse, (dq, dk, dv) = _run(q, k, v, g, 8.0)
    _is_value("out", out, v[:, top:top + 1], scores[top].item())
    assert (lse == scores[top].item()).all() or scores[top] == 0
    gd = g.double().cpu()[0, :, 0]
    ref.check("d_v", dv[:, top, 0], gd.sum(0)[None], (2 * Lq + 16) * EPS * gd.abs().sum(0)[None] + rounded(gd.sum(0)[None], dtype))
    rest = torch.arange(Lk) != top
    assert not dv[0, rest].any() and not dk[0, rest].any() and dq.isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Lq", ROWS)
@pytest.mark.parametrize("S", [0.0, 2.0 ** 14, 2.0 ** 17, -2.0 ** 18])
def test_small_differences_of_far_scores(S, Lq, dtype):
    """S + t, t multiples of 1 / 8 up to 12: weights as of t alone; the gradient as exact as lse is."""
    new = _gen(Lq + 9)
    Lk, D = 700, 64
    v, g = new(1, Lk, 1, D, dtype=dtype), new(1, Lq, 1, D, sigma=0.3, dtype=dtype)
    t = ((torch.arange(Lk) * 389) % 97).double() / 8
    t[5:] -= 4
    by = 512.0
    q, k = torch.zeros(D, dtype=torch.float64), torch.zeros(Lk, D, dtype=torch.float64)
    q[0], q[1], k[:, 0], k[:, 1] = by, 1.0, S / by, t
    q, k = q.to(dtype).cuda().expand(1, Lq, 1, D).contiguous(), k.to(dtype).cuda().view(1, Lk, 1, D)
    assert torch.equal(k[0, :, 0, 1].double().cpu(), t)
    out, lse, grads = _run(q, k, v, g, 1.0)
    p = torch.softmax(t, 0)
    w = (8 * ((t - t.max()).abs() + 1) + 6 * (Lk / 16 + 1)) * EPS
    vd = v[0, :, 0].double().cpu()
    want = p @ vd
    half = 0.0 if dtype == F32 else U[dtype]
    e = (p * (w + half)) @ vd.abs() + want.abs() * (p * w).sum() + (4 * Lk + 16) * EPS * (p @ vd.abs()) + rounded(want, dtype)
    if dtype == F16:
        e = e + ref.FLOOR * vd.abs().sum(0)
    ref.check("out", out[0, :, 0], want.expand(Lq, D), 1.01 * e.expand(Lq, D))
    exact = S + torch.logsumexp(t, 0)
    assert ((lse.double().cpu() - exact).abs() <= (p * w).sum() + (2 * Lk + 20) * EPS + 2 * EPS * abs(S)).all()
    # the gradient's bounds with what the stored lse is off by in place of 8 EPS |lse|
    off = (lse.double().cpu() - exact).abs().max().item() + (FAR_ROUNDING if abs(S) < 256 else 0)
    gd = g.double().cpu()[0, :, 0]
    o = want
    rel = w + off + EPS
    dp = gd @ vd.t()
    delta = gd @ o
    e_dp = (2 * D + 8) * EPS * (gd.abs() @ vd.abs().t())
    e_delta = gd.abs() @ (1.01 * e) + (2 * D + 8) * EPS * (gd.abs() @ o.abs())
    ds = p * (dp - delta[:, None])
    e_ds = p * (rel * (dp - delta[:, None]).abs() + e_dp + e_delta[:, None]) * (1 + rel) + 4 * EPS * ds.abs()
    e_ds = e_ds + half * (ds.abs() + e_ds)
    e_p = p * (rel + half)
    if dtype == F16:
        size = ds.abs() + e_ds
        e_ds = e_ds + ref.FLOOR * torch.maximum(size.amax(1, keepdim=True), size.amax(0, keepdim=True))
        e_p = e_p + ref.FLOOR
    kd, qd = k[0, :, 0].double().cpu(), q[0, :, 0].double().cpu()
    for name, got, a, b, ea, terms in (("d_q", grads[0], ds, kd, e_ds, Lk), ("d_k", grads[1], ds.t(), qd, e_ds.t(), Lq),
                                       ("d_v", grads[2], p.expand(Lq, Lk).t(), gd, e_p.expand(Lq, Lk).t(), Lq)):
        val = a @ b
        bound = ea @ b.abs() + (4 * terms + 16) * EPS * ((a.abs() + ea) @ b.abs()) + 4 * EPS * val.abs()
        ref.check(name, got[0, :, 0], val, 1.02 * bound + rounded(val, dtype))


#: below |lse| = 256 the weights' exponent is made from lse log2 e: its roundings there, in powers of e
FAR_ROUNDING = 4 * EPS * 256
