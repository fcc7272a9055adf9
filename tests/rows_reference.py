"""The row operators (include/corr.h, "Rows") in float64, and how far the library's results may be from them.

Rounding to a type is off by at most U = half its eps, relative to the value.  Everything between load and store is fp32, EPS = 2^-24 an
operation; a bound below counts the operations that reach a result and multiplies by the sum of the magnitudes they act on.

linear.  z is a sum of K products, S = sum |x w| + |b|; added in any order the sum is off by (K + 1) EPS S at most.  fp32 operands are
    three bf16 parts each: |a2| <= 2^-8 |a|, |a3| <= 2^-16 |a|, remainder 2^-24 |a|; the products left out are 4 EPS S at most, the six
    kept are 6 K terms.  The matrix instruction may cut where it aligns its terms: twice the bound, (2 K + 8) EPS S for 16-bit
    operands and (12 K + 16) EPS S for fp32.  Activations: slope at most 1.13 (silu 1.0999, gelu 1.129), the function itself
    16 EPS (|z| + 1): erff, expf, reciprocal and three products.
gradient.  dz = dy act'(z): 16 EPS |dy| (2 + |z|), and for 16-bit types with an activation U |dz| more.  d_x, d_w: sums of N, M products.
norms.  A row's sum goes through at most 32 additions (16 in a thread, 10 over lanes and waves, 6 spare): mean and square sum
    are 32 EPS off, relative to the sum of magnitudes; the normalised element 64 EPS (|hat| + rho mean|v|).  A chain of
    normalise, scale, add, normalise doubles that; NORM_OPS = 256 covers the forward pass and the gradient's two passes each.
"""
import math

import torch

EPS = 2.0 ** -24
NORM_OPS = 256
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
#: what rounding to the type adds near zero (half the smallest subnormal)
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid")


def act(name, z):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return torch.sigmoid(z) if name == "sigmoid" else z


def slope(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    z = z.detach().clone().requires_grad_()
    act(name, z).sum().backward()
    return z.grad


def rounded(value, dtype):
    """How far a value that is rounded once may be off."""
    return U[dtype] * value.abs() + TINY[dtype]


def linear(x, w, b, name, res):
    """(y, z, bound of y, bound of z) for operands of x's type."""
    dtype, K = x.dtype, x.shape[1]
    x, w = x.double().cpu(), w.double().cpu()
    z = x @ w.t()
    S = x.abs() @ w.abs().t()
    if b is not None:
        z, S = z + b.double().cpu(), S + b.double().cpu().abs()
    y = act(name, z)
    ops = 12 * K + 16 if dtype == torch.float32 else 2 * K + 8
    ez = ops * EPS * S
    ey = 1.13 * ez + (16 * EPS * (z.abs() + 1) if name != "none" else 0)
    if res is not None:
        r = res.double().cpu()
        y, ey = y + r, ey + EPS * (y.abs() + r.abs())
    return y, z, 1.01 * ey + rounded(y, dtype), 1.01 * ez + rounded(z, dtype)


def linear_backward(x, w, dy, z, name):
    """((d_x, bound), (d_w, bound), (d_b, bound))"""
    dtype, (M, K), N = x.dtype, x.shape, w.shape[0]
    x, w, dy = x.double().cpu(), w.double().cpu(), dy.double().cpu()
    dz, e = dy, torch.zeros_like(dy)
    if name != "none":
        z = z.double().cpu()
        dz = dy * slope(name, z)
        e = 16 * EPS * dy.abs() * (2 + z.abs())
    per = 12 if dtype == torch.float32 else 2
    ep = e + (rounded(dz, dtype) if name != "none" and dtype != torch.float32 else 0)

    def product(a, b, ea, terms):
        v, S = a @ b, a.abs() @ b.abs()
        return v, 1.01 * (ea @ b.abs() + (per * terms + 16) * EPS * S) + rounded(v, dtype)
    db = dz.sum(0)
    return (product(dz, w, ep, N), product(dz.t(), x, ep.t(), M),
            (db, 1.01 * (e.sum(0) + (M + 8) * EPS * dz.abs().sum(0)) + rounded(db, torch.float32)))


def _stats(v, kind, eps):
    if kind == "none":
        return v, torch.ones_like(v[:, :1]), v.abs()
    if kind == "layer":
        mean = v.mean(1, keepdim=True)
        rho = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)
        return (v - mean) * rho, rho, rho * (v.abs() + v.abs().mean(1, keepdim=True))
    rho = 1 / torch.sqrt((v ** 2).mean(1, keepdim=True) + eps)
    return v * rho, rho, rho * v.abs()


class Norm:
    """corr_residual_norm's arguments in float64: forward() and backward() give lists of (value, bound)."""

    def __init__(self, h, y, gate, gate_act, s, alpha, post, w1, b1, pre, w2, b2, eps, dtype):
        self.S, self.T = h.dtype, dtype
        d = lambda t: None if t is None else t.double().cpu()  # noqa: E731
        h, y, gate, s, w1, b1, w2, b2 = map(d, (h, y, gate, s, w1, b1, w2, b2))
        C = h.shape[1]
        one, zero = torch.ones(C, dtype=torch.float64), torch.zeros(C, dtype=torch.float64)
        self.has = [v is not None for v in (s, w1, b1, w2, b2)]
        self.s, self.w1, self.b1, self.w2, self.b2 = (one if s is None else s, one if w1 is None else w1, zero if b1 is None else b1,
                                                      one if w2 is None else w2, zero if b2 is None else b2)
        self.post, self.pre, self.alpha, self.block, self.gate_act = post, pre, alpha if y is not None else 1.0, y is not None, gate_act
        self.gate = gate
        if self.block:
            self.hat1, self.rho1, m1 = _stats(y, post, eps)
            self.p = self.hat1 * self.w1 + self.b1
            self.mp = m1 * self.w1.abs() + self.b1.abs()              # magnitudes that reach p
            self.m1 = m1
            self.a = act(gate_act, gate) if gate is not None else torch.ones_like(y)
            self.ma = self.a.abs() + (gate.abs() * 0.1 + 0.1 if gate is not None else 0)
            self.t = alpha * h + self.s * self.a * self.p
            self.mt = (alpha * h).abs() + self.s.abs() * self.ma * self.mp
        else:
            self.t, self.mt = h, h.abs()
        self.hat2, self.rho2, _ = _stats(self.t, pre, eps)
        if pre != "none":
            # an error of t moves the normalised row by rho times it, by its mean, and along the row
            e = self.mt
            self.m2 = self.rho2 * (e + e.mean(1, keepdim=True)) + self.hat2.abs() * (self.rho2 * (e * self.hat2.abs()).mean(1, keepdim=True) + 1)

    def forward(self):
        out = [(self.t, NORM_OPS * EPS * self.mt + rounded(self.t, self.S))] if self.block else []
        if self.pre != "none":
            n = self.hat2 * self.w2 + self.b2
            out.append((n, 2 * NORM_OPS * EPS * (self.m2 * self.w2.abs() + self.b2.abs()) + rounded(n, self.T)))
        return out

    @staticmethod
    def _back(q, mq, hat, mhat, rho, kind):
        if kind == "none":
            return q, mq
        C = q.shape[1]
        along = (q * hat).sum(1, keepdim=True) / C
        malong = (mq * mhat).sum(1, keepdim=True) / C
        mean, mmean = (q.sum(1, keepdim=True) / C, mq.sum(1, keepdim=True) / C) if kind == "layer" else (0.0, 0.0)
        return rho * (q - mean - hat * along), rho * (mq + mmean + mhat * malong)

    def backward(self, dh, dn):
        """(d_h, d_y, d_gate, d_scale, d_w1, d_b1, d_w2, d_b2), None for what is absent.  A magnitude (m...) is what the value
        would be if nothing cancelled; every step between adds at most NORM_OPS roundings of it."""
        c = 4 * NORM_OPS * EPS
        zero = torch.zeros_like(self.t)
        D, mD = (zero, zero) if dh is None else (dh.double().cpu(), dh.double().cpu().abs())
        dw2 = db2 = (torch.zeros(self.t.shape[1], dtype=torch.float64),) * 2
        if dn is not None:
            dn = dn.double().cpu()
            mhat = self.m2
            q, mq = self._back(dn * self.w2, (dn * self.w2).abs(), self.hat2, mhat, self.rho2, self.pre)
            # rho2 and hat2 carry t's error too
            D, mD = D + q, mD + mq * (1 + (self.rho2 * self.mt).mean(1, keepdim=True))
            dw2, db2 = self._column(dn * self.hat2, c * dn.abs() * mhat), self._column(dn, zero)
        out = [(self.alpha * D, c * mD * abs(self.alpha) + rounded(self.alpha * D, self.S)), None, None, None, None, None, None, None]
        if self.has[3]:
            out[6] = dw2
        if self.has[4]:
            out[7] = db2
        if not self.block:
            return out
        u, mu = D * self.s, mD * self.s.abs()
        dp, mdp = u * self.a, mu * self.ma
        if self.gate is not None:
            sl = slope(self.gate_act, self.gate)
            g = u * self.p * sl
            out[2] = (g, c * mu * self.mp * (sl.abs() + 0.1 * (1 + self.gate.abs())) + rounded(g, self.T))
        dy, mdy = self._back(dp * self.w1, mdp * self.w1.abs(), self.hat1, self.m1, self.rho1, self.post)
        out[1] = (dy, c * mdy + rounded(dy, self.T))
        if self.has[0]:
            out[3] = self._column(D * self.a * self.p, c * mD * self.ma * self.mp)
        if self.has[1]:
            out[4] = self._column(dp * self.hat1, c * mdp * self.m1)
        if self.has[2]:
            out[5] = self._column(dp, c * mdp)
        return out

    @staticmethod
    def _column(v, e):
        total = v.sum(0)
        return total, e.sum(0) + (v.shape[0] + 16) * EPS * v.abs().sum(0) + rounded(total, torch.float32)


def check(name, got, want, bound):
    """Every element within its bound; prints the largest share of it."""
    got = got.detach().double().cpu().reshape(want.shape)
    off = (got - want).abs()
    share = float((off / bound.clamp_min(1e-300)).max()) if off.numel() else 0.0
    print("%s: largest error / bound %.3f" % (name, share), flush=True)
    assert torch.isfinite(got).all(), name
    assert share <= 1.0, (name, share)
