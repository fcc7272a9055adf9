"""The operators on maps (include/corr.h, "Maps") in float64, and how far the library's results may be from them.

U, EPS and `rounded` are rows_reference's: half a step of a type, 2^-24 an fp32 operation.  A sum of n products in any order is off by
(2 n + 8) EPS times the sum of the magnitudes (the matrix instruction may cut where it aligns its terms).

attention.  A score s = scale <q, k> is off by (2 D + 12) EPS S, S the magnitudes' sum.  A weight e^(s - m) is formed as 2^(s c - m c), c = scale log2 e: the
    roundings of c, m c, the exponent and the power are 8 EPS (|s| + |m| + 1), relative; m's own error is the row's and cancels.  Sums are rescaled
    when the maximum grows, at most once a tile of 16 keys: 2 EPS each, and the power's 4 EPS.  So a weight is off by w = (2 D + 12) EPS S +
    EPS (8 (|s| + |m| + 1) + 6 (Lk / 16 + 1)), relative, and as an operand by U (16-bit types; up to 512 rows by 2 U U, in two parts) more.  out = sum p v with sum p = 1:
    sum p (w + U) |v| + |out| sum p w + (4 Lk + 16) EPS sum p |v|; lse: sum p w + (2 Lk + 8) EPS + 8 EPS |lse|.
gradient.  P = e^(s - lse) with the lse that was stored (off by e_l): relative error w + e_l + 8 EPS |lse|.  dP: (2 D + 8) EPS sum |dO v|.  delta = sum dO out
    with the out that was stored: its bound times |dO|, and (2 D + 8) EPS sum |dO out|.  dS = P (dP - delta): P (rel |dP - delta| + e_dP +
    e_delta) + 4 EPS |P (dP - delta)|, and as an operand as the weights.  The three products are sums of Lk or rows terms.  fp16 keeps weights to 2^-39 of
    the largest and dS to 2^-39 of the row's (key's) largest: FLOOR.
    The power and the matrix instructions take values below fp32's normal ones (2^-126) as zero: a weight may be off by LEAST = 2^-126, dS by that
    times |dP - delta| and once more for its own product, and each term of a sum by LEAST.
"""
import torch

from rows_reference import EPS, TINY, U, check, rounded  # noqa: F401  (for the tests)

F32 = torch.float32
FLOOR = 2.0 ** -38
LEAST = 2.0 ** -126


def heads_of(x, per):
    """[B, L, HK, D] as float64 [B, HK * per, L, D]"""
    return x.double().cpu().transpose(1, 2).repeat_interleave(per, 1)


def valid_keys(B, Lk, k_lengths=None, key_mask=None):
    keep = torch.ones(B, Lk, dtype=torch.bool)
    if k_lengths is not None:
        keep &= torch.arange(Lk) < k_lengths.cpu()[:, None]
    if key_mask is not None:
        keep &= key_mask.cpu() != 0
    return keep


class Attention:
    def __init__(self, q, k, v, scale, k_lengths=None, key_mask=None):
        self.T = q.dtype
        (B, Lq, H, D), Lk = q.shape, k.shape[1]
        self.per, self.scale = H // k.shape[2], scale
        # in two parts up to 512 rows: the first, towards zero, leaves up to 2 U, of which the second is U off, and up to 2^-30 (fp16: half of FLOOR) more is
        # added: (2 U + 2^-30) U + 2^-30
        few = B * Lq * H <= 512
        self.lp = 0.0 if self.T == F32 else 2 * U[self.T] ** 2 + 2.0 ** -29 if few else U[self.T]
        self.floor = 2 * FLOOR if few else FLOOR
        keep = valid_keys(B, Lk, k_lengths, key_mask)[:, None, None]
        clean = lambda t: torch.where(keep[:, 0, 0, :, None, None], t.cpu(), torch.zeros((), dtype=t.dtype))  # noqa: E731
        self.q, self.k, self.v = q.double().cpu().transpose(1, 2), heads_of(clean(k), self.per), heads_of(clean(v), self.per)
        s = scale * self.q @ self.k.transpose(2, 3)
        S = scale * self.q.abs() @ self.k.abs().transpose(2, 3)
        low = torch.full((), -float("inf"), dtype=torch.float64)
        s = torch.where(keep, s, low)
        if Lk:
            top = s.max(3, keepdim=True).values
        else:
            top = torch.full(s.shape[:3] + (1,), -float("inf"), dtype=torch.float64)
        top = torch.where(top == low, 0.0, top)
        p = torch.exp(s - top)
        total = p.sum(3, keepdim=True)
        self.lse = (total.log() + top)[..., 0]
        self.p = p / torch.where(total == 0, 1.0, total)
        size = torch.where(keep, s.abs(), 0.0)
        self.w = (2 * D + 12) * EPS * S + EPS * (8 * (size + top.abs() + 1) + 6 * (Lk / 16 + 1))
        self.s_size = size
        self.out = self.p @ self.v
        av = self.v.abs()
        pw = (self.p * self.w).sum(3, keepdim=True)
        e = (self.p * (self.w + self.lp) + LEAST) @ av + self.out.abs() * pw + (4 * Lk + 16) * EPS * (self.p @ av) + Lk * LEAST
        if self.T == torch.float16:
            e = e + self.floor * keep.double().expand_as(self.p) @ av
        self.e_out = 1.01 * e + rounded(self.out, self.T)
        finite = torch.where(self.lse == low, 0.0, self.lse)
        self.finite = finite[..., None]
        self.e_lse = 1.01 * (pw[..., 0] + (2 * Lk + 8) * EPS + 8 * EPS * finite.abs()) + rounded(finite, F32)

    def forward(self):
        """(out, bound) as [B, Lq, H, D], (lse, bound) as [B, H, Lq]"""
        return (self.out.transpose(1, 2), self.e_out.transpose(1, 2)), (self.lse, self.e_lse)

    def backward(self, d_out):
        """((d_q, bound), (d_k, bound), (d_v, bound)) laid out as the arguments"""
        g = d_out.double().cpu().transpose(1, 2)
        D, Lq, Lk, scale = g.shape[3], g.shape[2], self.k.shape[2], self.scale
        rel = self.w + self.e_lse[..., None] + 8 * EPS * self.finite.abs()
        dp = g @ self.v.transpose(2, 3)
        delta = (g * self.out).sum(3, keepdim=True)
        e_dp = (2 * D + 8) * EPS * (g.abs() @ self.v.abs().transpose(2, 3))
        e_delta = (g.abs() * self.e_out).sum(3, keepdim=True) + (2 * D + 8) * EPS * (g.abs() * self.out.abs()).sum(3, keepdim=True)
        ds = self.p * (dp - delta)
        e_ds = self.p * (rel * (dp - delta).abs() + e_dp + e_delta) * (1 + rel) + 4 * EPS * ds.abs()
        e_ds = e_ds + self.lp * (ds.abs() + e_ds) + LEAST * (1 + (dp - delta).abs())
        e_p = self.p * (rel + self.lp) + LEAST
        if self.T == torch.float16 and Lk and Lq:
            size = (ds.abs() + e_ds)
            e_ds = e_ds + FLOOR * torch.maximum(size.max(3, keepdim=True).values, size.max(2, keepdim=True).values)
            e_p = e_p + self.floor

        def product(a, b, ea, terms, by):
            v = by * (a @ b)
            bound = by * (ea @ b.abs() + (4 * terms + 16) * EPS * ((a.abs() + ea) @ b.abs()) + terms * LEAST)
            return v, 1.01 * bound + 4 * EPS * v.abs()

        def shared(t):                                  # [B, H, Lk, D] summed over the heads that share a key head
            return t.unflatten(1, (-1, self.per)).sum(2).transpose(1, 2)
        dq, eq = product(ds, self.k, e_ds, Lk, scale)
        n = Lq * self.per
        dk, ek = (shared(t) for t in product(ds.transpose(2, 3), self.q, e_ds.transpose(2, 3), n, scale))
        dv, ev = (shared(t) for t in product(self.p.transpose(2, 3), g, e_p.transpose(2, 3), n, 1.0))
        return ((dq.transpose(1, 2), (eq + rounded(dq, self.T)).transpose(1, 2)), (dk, ek + rounded(dk, self.T)), (dv, ev + rounded(dv, self.T)))


class GroupNorm:
    """Means and squares are merged along a chain: at most 16 chunks of a thread, 8 steps over threads, and P C / G / 2048 + 9 of a group's parts, of three
    operations each: OPS of them, relative to the largest magnitude for the mean; the squares are of differences whose own error is that of the
    mean.  Sums over rows go through at most P / 8 + 64 additions.  relu's slope may fall on either side where |z| is within its error."""

    def __init__(self, x, G, w, b, name, eps):
        self.T, self.name, self.G, self.wide = x.dtype, name, G, x.shape[2]
        x = x.double().cpu()
        B, P, C = x.shape
        one, zero = torch.ones(C, dtype=torch.float64), torch.zeros(C, dtype=torch.float64)
        by = lambda v: v.view(G, C // G)  # noqa: E731
        self.w, self.b = by(one if w is None else w.double().cpu()), by(zero if b is None else b.double().cpu())
        x = x.view(B, P, G, C // G)
        self.n = P * (C // G)
        mean = x.mean((1, 3), keepdim=True)
        var = ((x - mean) ** 2).mean((1, 3), keepdim=True)
        rho = 1 / torch.sqrt(var + eps)
        ops = 3 * (33 + self.n / 2048)
        most = x.abs().amax((1, 3), keepdim=True)
        e_mean = ops * EPS * most
        e_var = ops * EPS * (var + 2 * most * var.sqrt() + ops * EPS * most ** 2)
        e_rho = rho * (0.5 * e_var / (var + eps) + 4 * EPS)
        self.hat, self.rho, self.P = (x - mean) * rho, rho, P
        self.e_hat = (x - mean).abs() * e_rho + (rho + e_rho) * (e_mean + EPS * (x.abs() + mean.abs()))
        self.e_rho = e_rho
        self.z = self.hat * self.w + self.b
        self.e_z = self.w.abs() * self.e_hat + 4 * EPS * ((self.hat * self.w).abs() + self.b.abs())
        self.stats = torch.cat([mean, rho], 3).view(B, G, 2)
        self.e_stats = 1.01 * torch.cat([e_mean, e_rho], 3).view(B, G, 2) + EPS * self.stats.abs()

    def _flat(self, v):
        return v.reshape(v.shape[0], v.shape[1], self.wide)

    def forward(self):
        from rows_reference import act
        y = act(self.name, self.z)
        e = 1.13 * self.e_z + (16 * EPS * (self.z.abs() + 1) if self.name != "none" else 0)
        return (self._flat(y), self._flat(1.01 * e + rounded(y, self.T))), (self.stats, self.e_stats)

    def backward(self, d_y):
        from rows_reference import slope
        g = d_y.double().cpu().view(self.z.shape)
        e_slope = torch.zeros_like(g)
        if self.name == "relu":
            e_slope = (self.z.abs() <= self.e_z).double()
        elif self.name != "none":
            e_slope = 16 * EPS * (2 + self.z.abs()) + 1.2 * self.e_z
        dz = g * slope(self.name, self.z)
        e_dz = g.abs() * (e_slope + EPS)
        chain = (self.P / 8 + 64) * EPS

        def total(v, e, dims):
            return v.sum(dims, keepdim=True), e.sum(dims, keepdim=True) + chain * (v.abs() + e).sum(dims, keepdim=True)
        h, e_h = dz * self.hat, e_dz * (self.hat.abs() + self.e_hat) + dz.abs() * self.e_hat
        q, e_q = dz * self.w, (e_dz + EPS * dz.abs()) * self.w.abs()
        qh, e_qh = h * self.w, (e_h + 2 * EPS * h.abs()) * self.w.abs()
        s1, e1 = total(q, e_q, (1, 3))
        s2, e2 = total(qh, e_qh, (1, 3))
        n = self.n
        inner = q - s1 / n - self.hat * s2 / n
        size = q.abs() + s1.abs() / n + (self.hat * s2).abs() / n
        e_inner = e_q + (e1 + self.hat.abs() * e2 + self.e_hat * (s2.abs() + e2)) / n + 8 * EPS * size
        dx = self.rho * inner
        e_dx = self.rho * e_inner + (inner.abs() + e_inner) * self.e_rho + 2 * EPS * dx.abs()
        out = [(self._flat(dx), self._flat(1.01 * e_dx + rounded(dx, self.T)))]
        for v, e in ((h, e_h), (dz, e_dz)):
            s, es = total(v, e, (0, 1))
            out.append((s.reshape(-1), (1.01 * es + rounded(s, F32)).reshape(-1)))
        return out


def _gated_ops(dtype, K):
    return 12 * K + 16 if dtype == F32 else 2 * K + 8


def gated(x, w, b, name):
    """(y, z, bound of y, bound of z) of corr_gated_linear: the sums as rows_reference's linear, the activation off by 16 EPS (|gate| + 1) with a slope of
    at most 1.13, and their product."""
    from rows_reference import act
    dtype, N = x.dtype, w.shape[0] // 2
    x, w = x.double().cpu(), w.double().cpu()
    z, S = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        z, S = z + b.double().cpu(), S + b.double().cpu().abs()
    ez = _gated_ops(dtype, x.shape[1]) * EPS * S
    gate, up = z[:, :N], z[:, N:]
    a = act(name, gate)
    ea = 1.13 * ez[:, :N] + (16 * EPS * (gate.abs() + 1) if name != "none" else 0)
    y = a * up
    ey = ea * (up.abs() + ez[:, N:]) + a.abs() * ez[:, N:] + 2 * EPS * y.abs()
    return y, z, 1.01 * ey + rounded(y, dtype), 1.01 * ez + rounded(z, dtype)


def gated_backward(x, w, dy, z, name):
    """((d_x, bound), (d_w, bound), (d_b, bound)).  dz as an operand: bf16 rounded once, up to M min(N, K)
    = 2048 in two parts (U U, and the low part's own 2^-126), fp16 in two parts of 22 bits together with a floor of 2^-36."""
    from rows_reference import act, slope
    dtype, (M, K), N = x.dtype, x.shape, w.shape[0] // 2
    x, w, dy, z = (t.double().cpu() for t in (x, w, dy, z))
    gate, up = z[:, :N], z[:, N:]
    far = 16 * EPS * (2 + gate.abs()) if name != "none" else 0
    dz = torch.cat([dy * up * slope(name, gate), dy * act(name, gate)], 1)
    e = torch.cat([(dy * up).abs() * far, dy.abs() * far], 1) + 3 * EPS * dz.abs()
    low = U[torch.bfloat16] ** 2 if M * min(N, K) <= 2048 else U[torch.bfloat16]
    ep = e + {F32: 0.0, torch.bfloat16: low, torch.float16: 2.0 ** -21}[dtype] * (dz.abs() + e)
    if dtype == torch.bfloat16:
        ep = ep + LEAST
    if dtype == torch.float16:
        ep = ep + 2.0 ** -35
    per = 12 if dtype == F32 else 2

    def product(a, b, ea, terms):
        v = a @ b
        return v, 1.01 * (ea @ b.abs() + (per * terms + 16) * EPS * ((a.abs() + ea) @ b.abs())) + rounded(v, dtype)
    db = dz.sum(0)
    return (product(dz, w, ep, 2 * N), product(dz.t(), x, ep.t(), M),
            (db, 1.01 * (e.sum(0) + (M + 8) * EPS * dz.abs().sum(0)) + rounded(db, F32)))
