"""corr_group_norm and its gradient on the GPU against float64: sizes around their threads' pieces, every activation, layouts, means far above the
spread, values that are not finite, graphs.  The bounds are derived in maps_reference.py."""
import itertools

import pytest

import maps_reference as ref
from rows_reference import ACTS, slope

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)
EPS = 1e-5


def _b():
    from paper_2505_16942_amd import binding
    return binding


def _act(name):
    return getattr(_b(), "CORR_ACT_" + name.upper())


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return lambda *shape, sigma=1.0, mean=0.0, dtype=F32: (torch.randn(shape, generator=g) * sigma + mean).to(dtype).cuda()


def _run(x, G, w, b, g, act, **kw):
    m = _b()
    stats = torch.full((x.shape[0], G, 2), float("nan"), device="cuda")
    y = m.corr_group_norm(x, G, weight=w, bias=b, act=act, eps=EPS, stats=stats, **kw)
    return y, stats, m.corr_group_norm_backward(x, G, stats, g, weight=w, bias=b, act=act)


def _compare(what, x, G, w, b, g, name):
    y, stats, grads = _run(x, G, w, b, g, _act(name))
    want = ref.GroupNorm(x, G, w, b, name, EPS)
    (wy, ey), (ws, es) = want.forward()
    ref.check(what + " y", y, wy, ey)
    ref.check(what + " stats", stats, ws, es)
    for n, got, (v, e) in zip(("d_x", "d_weight", "d_bias"), grads, want.backward(g)):
        ref.check("%s %s" % (what, n), got, v, e)
    return y, stats, grads


# (B, P, C, G): one element and few; a group, a channel and an item at a time; odd everything; pieces that end inside a row; several columns of workgroups
SIZES = [(1, 1, 1, 1), (2, 1, 8, 2), (1, 7, 3, 1), (3, 50, 24, 8), (1, 2852, 64, 8), (2, 333, 96, 32), (1, 4097, 256, 32), (4, 65, 130, 13), (1, 100, 3, 3),
         (2, 40, 2056, 8), (1, 30, 16384, 64), (1, 5, 4100, 4100), (5, 1000, 5, 1), (1, 9, 17, 17), (300, 6, 16, 4), (2, 64, 128, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_group_norm(size, dtype):
    m, (B, P, C, G) = _b(), size
    new = _gen(B + 3 * P + 5 * C + 7 * G)
    x = new(B, P, C, mean=0.5, dtype=dtype)
    w, b = (new(C, sigma=0.3, mean=1.0), new(C, sigma=0.3)) if (B + P + G) % 4 else (None, None)
    g, name = new(B, P, C, sigma=0.3, dtype=dtype), ACTS[(P + C) % 6]
    y, stats, grads = _compare("%s %s %s" % (size, dtype, name), x, G, w, b, g, name)
    again = _run(x, G, w, b, g, _act(name))
    assert torch.equal(y, again[0]) and torch.equal(stats, again[1]) and all(torch.equal(p, q) for p, q in zip(grads, again[2])), "two calls differ"
    assert torch.equal(y, m.corr_group_norm(x, G, weight=w, bias=b, act=_act(name), eps=EPS)), "without stats"
    for want in itertools.product((False, True), repeat=3):
        part = m.corr_group_norm_backward(x, G, stats, g, weight=w, bias=b, act=_act(name), want_x=want[0], want_weight=want[1], want_bias=want[2])
        for p, q, wanted in zip(part, grads, want):
            assert (p is None) if not wanted else torch.equal(p, q)


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations(name, dtype):
    new = _gen(4)
    x, g = new(2, 300, 48, dtype=dtype), new(2, 300, 48, dtype=dtype)
    _compare("%s %s" % (name, dtype), x, 6, new(48, sigma=3.0), new(48), g, name)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_maps(dtype):
    """Enough rows that a thread merges many chunks: the statistics and sums against float64, some rows of the rest."""
    m, new = _b(), _gen(5)
    B, P, C, G = 2, 135 * 240, 72, 9
    x = torch.randn(B, P, C, device="cuda").to(dtype)
    g = torch.randn(B, P, C, device="cuda").mul_(0.1).to(dtype)
    w, b = new(C, mean=1.0, sigma=0.1), new(C, sigma=0.1)
    y, stats, grads = _run(x, G, w, b, g, m.CORR_ACT_SILU)
    want = ref.GroupNorm(x, G, w, b, "silu", EPS)
    (wy, ey), (ws, es) = want.forward()
    ref.check("y", y, wy, ey)
    ref.check("stats", stats, ws, es)
    for n, got, (v, e) in zip(("d_x", "d_weight", "d_bias"), grads, want.backward(g)):
        ref.check(n, got, v, e)


def test_means_far_above_the_spread():
    """fp32 rows around 4096 with a spread of one: the squares are taken about the mean."""
    new = _gen(6)
    x, g = new(2, 1000, 32, mean=4096.0), new(2, 1000, 32)
    y, stats, _ = _compare("far", x, 4, new(32, mean=1.0), new(32), g, "none")
    assert (stats[..., 1] > 0.5).all() and (stats[..., 1] < 2).all()
    for value in (3e20, 3e38):                                  # squares and sums overflow, differences are zero
        for P in (500, 50000):
            x = torch.full((1, P, 8), value, device="cuda")
            stats = torch.empty(1, 2, 2, device="cuda")
            assert not _b().corr_group_norm(x, 2, stats=stats).any() and (stats[..., 0] == x[0, 0, 0]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Columns of wider rows, a map of two axes, and in place: the same bits."""
    m, new = _b(), _gen(7)
    wide = new(2, 6, 50, 3 * 40, dtype=dtype)
    x = wide[..., 40:80]
    w, b = new(40, mean=1.0), new(40)
    wide_g = new(2, 300, 41, dtype=dtype)
    g = wide_g[..., :40]
    want = _run(x.contiguous().view(2, 300, 40), 5, w, b, g.contiguous(), m.CORR_ACT_RELU)
    got = _run(x, 5, w, b, g, m.CORR_ACT_RELU)
    assert got[0].shape == x.shape and torch.equal(got[0].view(2, 300, 40), want[0]) and torch.equal(got[1], want[1])
    assert all(torch.equal(p.view(q.shape), q) for p, q in zip(got[2], want[2]))
    odd = new(2 * 300 * 40 + 1, dtype=dtype)[1:].view(2, 300, 40)            # begins on an odd element
    odd.copy_(x.reshape(2, 300, 40))
    got = _run(odd, 5, w, b, g, m.CORR_ACT_RELU)
    assert torch.equal(got[0], want[0]) and all(torch.equal(p, q) for p, q in zip(got[2], want[2]))
    y = m.corr_group_norm(odd, 5, weight=w, bias=b, act=m.CORR_ACT_RELU, out=odd)
    assert y is odd and torch.equal(y, want[0])
    with pytest.raises(ValueError):
        m.corr_group_norm(new(2, 8, 40, 40, dtype=dtype)[:, :5], 5)          # items not evenly spaced


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_finite(dtype):
    """A NaN or infinity stays in its item and group."""
    m, new = _b(), _gen(8)
    x, g = new(3, 200, 24, dtype=dtype), new(3, 200, 24, dtype=dtype)
    clean = _run(x, 4, None, None, g, m.CORR_ACT_RELU)
    for junk in (float("nan"), float("inf")):
        bad = x.clone()
        bad[1, 77, 13] = junk
        y, stats, (dx, dw, db) = _run(bad, 4, None, None, g, m.CORR_ACT_NONE)
        assert stats[1, 2].isnan().any() and y[1, :, 12:18].isnan().all() and dx[1, :, 12:18].isnan().all()
        y = m.corr_group_norm(bad, 4, act=m.CORR_ACT_RELU)
        keep = torch.ones_like(x, dtype=torch.bool)
        keep[1, :, 12:18] = False
        assert torch.equal(y[keep], clean[0][keep])


def test_differences():
    """The gradient against differences of the forward call in fp32: what the quotient itself is off by is computed in float64."""
    m, new = _b(), _gen(9)
    x, w, b, v = new(2, 30, 12), new(12, mean=1.0, sigma=0.2), new(12), new(2, 30, 12)
    _, _, grads = _run(x, 3, w, b, v, m.CORR_ACT_SILU)
    h = 2.0 ** -6
    for i, t in enumerate((x, w, b)):
        step = new(*t.shape)
        sides, exact, noise = [], [], 0.0
        for sign in (1.0, -1.0):
            args = [x, w, b]
            args[i] = t + sign * h * step
            sides.append((m.corr_group_norm(args[0], 3, weight=args[1], bias=args[2], act=m.CORR_ACT_SILU, eps=EPS).double() * v.double()).sum().item())
            wy, ey = ref.GroupNorm(args[0], 3, args[1], args[2], "silu", EPS).forward()[0]
            exact.append((wy * v.double().cpu()).sum().item())
            noise += (ey * v.double().cpu().abs()).sum().item()
        along, e = ref.GroupNorm(x, 3, w, b, "silu", EPS).backward(v)[i]
        true = (along * step.double().cpu()).sum().item()
        got = (grads[i].double() * step.double()).sum().item()
        truncation = abs((exact[0] - exact[1]) / (2 * h) - true)
        assert abs((sides[0] - sides[1]) / (2 * h) - got) <= truncation + noise / (2 * h) + (e * step.double().cpu().abs()).sum().item()
        assert truncation < 0.05 * abs(true) + 0.05


def test_graphs():
    m = _b()
    B, P, C, G = 2, 700, 40, 5
    x, g = _gen(10)(B, P, C, dtype=BF16), _gen(11)(B, P, C, dtype=BF16)
    w, b = _gen(12)(C), _gen(13)(C)
    y, stats, dx = torch.empty_like(x), torch.empty(B, G, 2, device="cuda"), torch.empty_like(x)
    dw, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    wf = torch.empty(m.corr_group_norm_workspace_bytes(BF16, B, P, C, G), dtype=torch.uint8, device="cuda")
    wb = torch.empty(m.corr_group_norm_backward_workspace_bytes(BF16, B, P, C, G), dtype=torch.uint8, device="cuda")

    def step():
        m.corr_group_norm(x, G, weight=w, bias=b, act=m.CORR_ACT_GELU, stats=stats, out=y, workspace=wf)
        m.corr_group_norm_backward(x, G, stats, g, weight=w, bias=b, act=m.CORR_ACT_GELU, d_x=dx, d_weight=dw, d_bias=db, workspace=wb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        x.copy_(_gen(60 + turn)(B, P, C, dtype=BF16))
        want = _run(x, G, w, b, g, m.CORR_ACT_GELU)
        for t in (y, stats, dx, dw, db, wf, wb):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(stats, want[1]) and all(torch.equal(p, q) for p, q in zip((dx, dw, db), want[2])), turn


def test_nothing_to_do():
    m = _b()
    for B, P in ((0, 5), (3, 0)):
        x = torch.randn(B, P, 8, device="cuda")
        stats = torch.full((B, 2, 2), 7.0, device="cuda")
        assert m.corr_group_norm(x, 2, stats=stats).shape == x.shape and not stats.any()
        dx, dw, db = m.corr_group_norm_backward(x, 2, stats, x)
        assert dx.shape == x.shape and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(16384, 3, 256, 256), (65535, 2, 128, 64), (65535, 2, 128, 128), (512, 16, 16384, 16384)])
def test_millions_of_groups(size, dtype):
    """2^22 items times groups and more, where a workgroup of 1024 threads each would be 2^32 threads: some items against float64, all of them written."""
    m, new, (B, P, C, G) = _b(), _gen(14), size
    x = torch.randn(B, P, C, device="cuda").to(dtype)
    g = torch.randn(B, P, C, device="cuda").mul_(0.1).to(dtype)
    w, b = new(C, mean=1.0, sigma=0.1), new(C, sigma=0.1)
    y, stats, (dx, dw, db) = _run(x, G, w, b, g, m.CORR_ACT_SILU)
    assert y.isfinite().all() and stats.isfinite().all() and (stats[..., 1] > 0).all() and dx.isfinite().all()
    some = torch.tensor([0, B // 2, B - 1], device="cuda")
    want = ref.GroupNorm(x[some], G, w, b, "silu", EPS)
    (wy, ey), (ws, es) = want.forward()
    ref.check("y", y[some], wy, ey)
    ref.check("stats", stats[some], ws, es)
    ref.check("d_x", dx[some], *want.backward(g[some])[0])
    # two channels' vectors: B items are up to B / 64 + 64 additions more
    W = C // G
    for c in (0, C - 1):
        lo = c // W * W
        cut = lambda t: t[..., lo:lo + W].contiguous()  # noqa: E731
        one = ref.GroupNorm(cut(x), 1, cut(w), cut(b), "silu", EPS)
        _, (v, e), (vb, eb) = one.backward(cut(g))
        dz = cut(g).double().cpu().view(one.z.shape) * slope("silu", one.z)
        more = (B / 64 + 64) * ref.EPS
        for what, got, val, bound, terms in (("d_weight", dw, v, e, dz * one.hat), ("d_bias", db, vb, eb, dz)):
            ref.check(what, got[lo:lo + W], val, bound + more * terms.abs().sum((0, 1)).reshape(-1))
    assert torch.equal(m.corr_group_norm(x, G, weight=w, bias=b, act=m.CORR_ACT_SILU, eps=EPS, out=x), y)


#: (B, P, C, G): a group in a workgroup's registers; sums by parts, of one group and of several; groups of three channels
MEANS = [(1, 8192, 4, 1), (2, 2048, 64, 8), (1, 50000, 8, 1), (2, 40000, 24, 8), (3, 9000, 96, 32)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", MEANS)
def test_a_value_far_from_the_others(size, dtype):
    """One value of 1e6 (6e4 in fp16) among ones of about one, first, last or anywhere: the mean is off by its sums' roundings, OPS of them relative to the mean of
    the magnitudes (a running mean's rounding counts as many values as it stands for), wherever the one lies."""
    m, (B, P, C, G) = _b(), size
    x = _gen(P + C)(B, P, C)
    ops = 3 * (33 + P * (C // G) / 2048) + 8
    for pixel, channel in ((0, 0), (P - 1, C - 1), (P // 3, C // 2)):
        x2 = x.clone()
        x2[:, pixel, channel] = 6e4 if dtype == F16 else 1e6
        x2 = x2.to(dtype)
        stats = torch.empty(B, G, 2, device="cuda")
        y = m.corr_group_norm(x2, G, eps=EPS, stats=stats)
        d = x2.double().cpu().view(B, P, G, C // G)
        mean, size = d.mean((1, 3), keepdim=True), d.abs().mean((1, 3), keepdim=True)
        rho = 1 / torch.sqrt(((d - mean) ** 2).mean((1, 3), keepdim=True) + EPS)
        e_mean = ops * ref.EPS * size + ref.EPS * mean.abs()
        ref.check("mean", stats[..., 0], mean.view(B, G), e_mean.view(B, G))
        want = (d - mean) * rho
        e = rho * e_mean + want.abs() * ops * ref.EPS + 4 * ref.EPS * rho * (d.abs() + mean.abs())
        ref.check("y", y, want.view(B, P, C), (1.01 * e + ref.rounded(want, dtype)).view(B, P, C))


@pytest.mark.parametrize("P", [500, 50000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_largest_values_of_either_sign(P, dtype):
    """Squares and differences that overflow: the normalised group is zero, with zero gradients."""
    m = _b()
    sign = (torch.rand(2, P, 16, generator=torch.Generator().manual_seed(P)) < 0.5).float().mul(2).sub(1)
    b = _gen(3)(16)
    for value in (2e38, 3.38e38):
        x = (sign * value).to(dtype).cuda()
        y, stats, (dx, dw, db) = _run(x, 2, None, b, torch.ones_like(x), m.CORR_ACT_NONE)
        assert torch.equal(y, b.to(dtype).expand_as(y)) and not stats.any()
        assert not dx.any() and not dw.any() and (db == 2 * P).all()


@pytest.mark.parametrize("P", [500, 50000])
def test_constants(P):
    """A group of one value has that value for its mean, whatever it is, and is zero when it is normalised."""
    m = _b()
    values = torch.rand(64, generator=torch.Generator().manual_seed(1)) + 1
    for scale in (1.0, 2.0 ** 20, 2.0 ** 127):
        x = (values * scale).clamp(max=3.4028234e38).cuda().view(1, 1, 64).repeat(1, P, 1)
        stats = torch.empty(1, 64, 2, device="cuda")
        y = m.corr_group_norm(x, 64, stats=stats)
        assert torch.equal(stats[0, :, 0], x[0, 0]) and not y.any()
        x = x.repeat_interleave(8, 2)
        stats = torch.empty(1, 64, 2, device="cuda")
        y = m.corr_group_norm(x, 64, stats=stats)
        assert torch.equal(stats[0, :, 0], x[0, 0, ::8]) and not y.any()


def test_sums_over_rows_in_the_2_norm():
    """Sums of normal terms in fp32.  A rounding is 0.41 * 2^-24 of what is rounded (rms), a chain of n additions so 0.41 * 2^-24 * sqrt(n / 2) of its sum, a tree of
    n levels 0.41 * 2^-24 * sqrt(n).  Eight rows a thread, trees over 8 threads and 64 shares, four items: 0.41 * 2^-24 * sqrt(4 + 9 + 2) = 9.5e-8; the
    terms (slope, hat and two products, about 4 * 2^-24 * 0.41) 9.8e-8; both 1.4e-7.  With the shares one after the other, sqrt(32) for sqrt(6): 1.9e-7."""
    m, new = _b(), _gen(15)
    B, P, C, G = 4, 7285, 96, 32
    x, g, w, b = new(B, P, C), new(B, P, C), new(C, mean=1.0, sigma=0.2), new(C, sigma=0.2)
    _, _, (_, dw, db) = _run(x, G, w, b, g, m.CORR_ACT_SILU)
    one = ref.GroupNorm(x, G, w, b, "silu", EPS)
    _, (vw, _), (vb, _) = one.backward(g)
    for got, want in ((dw, vw), (db, vb)):
        assert ((got.double().cpu() - want).norm() / want.norm()).item() < 1.6e-7
