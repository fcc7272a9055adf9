"""The row operators on the GPU against float64: every size class, type, activation, norm, layout and edge their kernels treat apart.
The bounds are derived in rows_reference.py."""
import itertools

import pytest

import rows_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)


def _b():
    from paper_2505_16942_amd import binding
    return binding


def _act(name):
    return getattr(_b(), "CORR_ACT_" + name.upper())


def _norm(name):
    return getattr(_b(), "CORR_NORM_" + name.upper())


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return lambda *shape, sigma=1.0, mean=0.0, dtype=F32: (torch.randn(shape, generator=g) * sigma + mean).to(dtype).cuda()


# (M, N, K): one element; few rows with whole, short and odd rows; one tile and its neighbours; a long k over few tiles; odd everything
SIZES = [(1, 1, 1), (1, 16, 32), (1, 300, 1000), (3, 5, 7), (16, 256, 324), (17, 33, 65), (32, 130, 512), (33, 64, 64), (64, 64, 324),
         (65, 126, 243), (129, 127, 81), (130, 1000, 36), (300, 8, 1024), (257, 257, 1100), (700, 256, 130), (40, 24, 4099),
         (100, 20, 3), (77, 1, 5), (2000, 1, 1), (1, 40, 9001), (32, 33, 2051), (20, 4100, 2100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_linear(size, dtype):
    b, (M, N, K) = _b(), size
    new = _gen(M * 7 + N * 3 + K)
    x, w = new(M, K, dtype=dtype), new(N, K, sigma=K ** -0.5, dtype=dtype)
    name = ref.ACTS[(M + N + K) % 6]
    bias = new(N, sigma=0.3) if (M + K) % 3 else None
    res = new(M, N, dtype=dtype) if (N + K) % 2 else None
    z = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
    y = b.corr_linear(x, w, bias=bias, act=_act(name), residual=res, preact=z)
    wy, wz, ey, ez = ref.linear(x, w, bias, name, res)
    assert y.dtype == dtype
    ref.check("y %s %s %s" % (size, dtype, name), y, wy, ey)
    ref.check("z", z, wz, ez)
    assert torch.equal(y, b.corr_linear(x, w, bias=bias, act=_act(name), residual=res)), "two calls differ"


@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations_far_out(name, dtype):
    """Every activation and slope on sums from -90 to 90."""
    b = _b()
    x = torch.linspace(-90, 90, 400).reshape(-1, 1).to(dtype).cuda()
    w = torch.ones(1, 1, dtype=dtype).cuda()
    y = b.corr_linear(x, w, act=_act(name))
    wy, _, ey, _ = ref.linear(x, w, None, name, None)
    ref.check("%s %s" % (name, dtype), y, wy, ey)
    dy = torch.ones_like(x)
    got = b.corr_linear_backward(x, w, dy, preact=x, act=_act(name))
    for g, (v, e), what in zip(got, ref.linear_backward(x, w, dy, x, name), ("d_x", "d_w", "d_b")):
        ref.check(what, g, v, e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_linear_backward(size, dtype):
    b, (M, N, K) = _b(), size
    new = _gen(M * 5 + N * 11 + K)
    x, w, dy = new(M, K, dtype=dtype), new(N, K, sigma=K ** -0.5, dtype=dtype), new(M, N, sigma=0.3, dtype=dtype)
    name = ref.ACTS[(M + N) % 6]
    z = new(M, N, dtype=dtype)
    got = b.corr_linear_backward(x, w, dy, preact=z if name != "none" else None, act=_act(name))
    for g, (v, e), what in zip(got, ref.linear_backward(x, w, dy, z, name), ("d_x", "d_w", "d_b")):
        ref.check("%s %s %s %s" % (what, size, dtype, name), g, v, e)
    again = b.corr_linear_backward(x, w, dy, preact=z if name != "none" else None, act=_act(name))
    assert all(torch.equal(p, q) for p, q in zip(got, again)), "two calls differ"
    for want in itertools.product((False, True), repeat=3):          # any subset gives the same bits
        part = b.corr_linear_backward(x, w, dy, preact=z if name != "none" else None, act=_act(name), want_x=want[0], want_w=want[1],
                                      want_bias=want[2])
        for p, q, wanted in zip(part, got, want):
            assert (p is None) if not wanted else torch.equal(p, q)


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_linear_large_tiles(dtype):
    """Sizes that fill the chip with the largest tiles, in each of the three layouts, with a ragged border and a short last step."""
    b, new = _b(), _gen(77)
    M, N, K = 4090, 4100, 72
    x, w, dy = new(M, K, dtype=dtype), new(N, K, sigma=0.1, dtype=dtype), new(M, N, dtype=dtype)
    ref.check("y", b.corr_linear(x, w), *(ref.linear(x, w, None, "none", None)[i] for i in (0, 2)))
    x2, w2 = dy.t().contiguous(), x                      # [4100, 4090] rows against [4090, 72]: d_w is [4090 .. ]
    x2, w2 = new(66, 4100, dtype=dtype), new(4090, 4100, sigma=0.02, dtype=dtype)
    dy2 = new(66, 4090, dtype=dtype)
    for g, (v, e), what in zip(b.corr_linear_backward(x2, w2, dy2), ref.linear_backward(x2, w2, dy2, None, "none"), ("d_x", "d_w", "d_b")):
        ref.check("wide " + what, g, v, e)
    x3, w3, dy3 = new(66000, 254, dtype=dtype), new(40, 254, dtype=dtype), new(66000, 40, dtype=dtype)
    for g, (v, e), what in zip(b.corr_linear_backward(x3, w3, dy3), ref.linear_backward(x3, w3, dy3, None, "none"), ("d_x", "d_w", "d_b")):
        ref.check("long " + what, g, v, e)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_short_sums_and_large_results(dtype):
    """Tiles for short sums (K up to 256, more than 128 columns, many rows), and results that go past the caches: rows here and there."""
    b, new = _b(), _gen(5)
    x, w, bias = new(66000, 70, dtype=dtype), new(131, 70, sigma=0.1, dtype=dtype), new(131)
    z = torch.empty(66000, 131, dtype=dtype, device="cuda")
    y = b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_SILU, preact=z)
    some = torch.cat([torch.arange(130), torch.arange(32700, 32900), torch.arange(65870, 66000)]).cuda()
    wy, wz, ey, ez = ref.linear(x[some], w, bias, "silu", None)
    ref.check("y", y[some], wy, ey)
    ref.check("z", z[some], wz, ez)
    M = (130 << 20) // 256 // x.element_size()
    x, w, res = new(M, 264, dtype=dtype), new(256, 264, sigma=0.1, dtype=dtype), new(M, 256, dtype=dtype)
    y = b.corr_linear(x, w, act=b.CORR_ACT_RELU, residual=res)
    some = torch.cat([torch.arange(260), torch.arange(M // 2, M // 2 + 100), torch.arange(M - 300, M)]).cuda()
    wy, _, ey, _ = ref.linear(x[some], w, None, "relu", res[some])
    ref.check("large", y[some], wy, ey)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [5, 90])
@pytest.mark.parametrize("K,ldx,ldy,ldr", [(40, 48, 64, 50), (40, 43, 35, 33), (39, 40, 32, 32)])
def test_linear_strides_and_guards(dtype, M, K, ldx, ldy, ldr):
    """Rows apart, odd strides, a result between others that stay as they were, and a residual that is the result."""
    b, new, N = _b(), _gen(K + ldx), 32
    xs, rs, dys = new(M, ldx, dtype=dtype), new(M, ldr, dtype=dtype), new(M, ldy, dtype=dtype)
    w = new(N, K, sigma=0.2, dtype=dtype)
    x, res, dy = xs[:, :K], rs[:, :N], dys[:, :N]
    wy, _, ey, _ = ref.linear(x, w, None, "silu", res)
    buf = torch.full((M + 2, ldy), 7.0, dtype=dtype, device="cuda")
    out = buf[1:M + 1, :N]
    b.corr_linear(x, w, act=b.CORR_ACT_SILU, residual=res, out=out)
    ref.check("strided", out, wy, ey)
    assert (buf[0] == 7).all() and (buf[M + 1] == 7).all() and (buf[:, N:] == 7).all()
    acc = rs.clone()
    b.corr_linear(x, w, act=b.CORR_ACT_SILU, residual=acc[:, :N], out=acc[:, :N])
    ref.check("in place", acc[:, :N], wy, ey)
    assert torch.equal(acc[:, N:], rs[:, N:])
    z = new(M, N, dtype=dtype)
    for g, (v, e), what in zip(b.corr_linear_backward(x, w, dy, preact=z, act=b.CORR_ACT_GELU),
                               ref.linear_backward(x, w, dy, z, "gelu"), ("d_x", "d_w", "d_b")):
        ref.check(what, g, v, e)
    for g, (v, e), what in zip(b.corr_linear_backward(x, w, dy), ref.linear_backward(x, w, dy, None, "none"), ("d_x", "d_w", "d_b")):
        ref.check(what + " plain", g, v, e)


def test_columns_of_one_buffer():
    """x, the residual and the results side by side in the rows of one buffer; columns that do meet are refused."""
    b, new = _b(), _gen(55)
    buf = new(50, 160, dtype=F16)
    w = new(32, 64, sigma=0.1, dtype=F16)
    x, res, out = buf[:, :64], buf[:, 64:96], buf[:, 96:128]
    keep = buf.clone()
    b.corr_linear(x, w, act=b.CORR_ACT_RELU, residual=res, out=out)
    wy, _, ey, _ = ref.linear(keep[:, :64], w, None, "relu", keep[:, 64:96])
    ref.check("out", out, wy, ey)
    assert torch.equal(buf[:, :96], keep[:, :96]) and torch.equal(buf[:, 128:], keep[:, 128:])
    for bad in (buf[:, 63:95], buf[:, 32:64], buf[:, 80:112]):
        with pytest.raises(b.CorrError):
            b.corr_linear(x, w, residual=res, out=bad)


def test_linear_shapes():
    """Leading dimensions, one row without any, no rows, evenly spaced views."""
    b, new = _b(), _gen(3)
    w = new(24, 81)
    x = new(2, 5, 7, 81)
    y = b.corr_linear(x, w)
    assert y.shape == (2, 5, 7, 24) and torch.equal(y.reshape(-1, 24), b.corr_linear(x.reshape(-1, 81), w))
    one = b.corr_linear(x[0, 0, 0], w)
    assert one.shape == (24,)
    ref.check("one row", one.reshape(1, -1), *(ref.linear(x[0, 0, 0].reshape(1, -1), w, None, "none", None)[i] for i in (0, 2)))
    # every second row is evenly spaced
    half = x[:, :, 0]
    assert torch.equal(b.corr_linear(half, w), b.corr_linear(half.contiguous(), w))
    with pytest.raises(ValueError):
        b.corr_linear(x[:, 1:3], w)                                  # two runs of rows with a gap of another size
    none = b.corr_linear(x[:0], w, bias=new(24))
    assert none.shape == (0, 5, 7, 24)
    for dtype in TYPES:
        e = torch.empty(0, 3, dtype=dtype, device="cuda")
        d_x, d_w, d_b = b.corr_linear_backward(e, new(5, 3, dtype=dtype), torch.empty(0, 5, dtype=dtype, device="cuda"),
                                               preact=torch.empty(0, 5, dtype=dtype, device="cuda"), act=b.CORR_ACT_RELU)
        assert d_x.shape == (0, 3) and (d_w == 0).all() and (d_b == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(4, 70), (70, 70), (70, 71), (300, 130)])
def test_linear_not_finite(dtype, M, K):
    """An infinity or NaN stays in its own row of the result, as in the sum itself, wherever its row ends inside a load of another."""
    b, new, N = _b(), _gen(M + K), 40
    x, w = new(M, K, dtype=dtype), new(N, K, dtype=dtype)
    x[1, 0], x[2, K - 1], x[3, 3], x[3, 4] = float("inf"), float("nan"), float("inf"), -float("inf")
    w[:, 3], w[:, 4] = w[:, 3].abs() + 0.5, w[:, 4].abs() + 0.5        # inf - inf
    y = b.corr_linear(x, w).double().cpu()
    want = x.double().cpu() @ w.double().cpu().t()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(y[1], want[1])                                  # infinities with their signs
    keep = [i for i in range(M) if i not in (1, 2, 3)]
    wy, _, ey, _ = ref.linear(x[keep], w, None, "none", None)
    ref.check("the other rows", y[keep], wy, ey)
    dy = new(M, N, dtype=dtype)
    dy[2, 5] = float("inf")
    d_x, d_w, _ = b.corr_linear_backward(new(M, K, dtype=dtype), w, dy)
    assert torch.isfinite(d_x).all(1).cpu().tolist() == [i != 2 for i in range(M)]
    assert torch.isfinite(d_w).all(1).cpu().tolist() == [n != 5 for n in range(N)]


def test_linear_odd_columns_beside_nan_in_the_workspace():
    """The gradient's own dz has rows with room behind them: what an earlier call left there reaches no result."""
    b, new = _b(), _gen(41)
    for dtype in TYPES:
        M, N, K = 300, 37, 70
        x, w, dy, z = new(M, K, dtype=dtype), new(N, K, sigma=0.1, dtype=dtype), new(M, N, dtype=dtype), new(M, N, dtype=dtype)
        ws = torch.full((b.corr_linear_backward_workspace_bytes(dtype, b.CORR_ACT_SILU, M, N, K),), 0xff, dtype=torch.uint8, device="cuda")
        got = b.corr_linear_backward(x, w, dy, preact=z, act=b.CORR_ACT_SILU, workspace=ws)
        for g, (v, e), what in zip(got, ref.linear_backward(x, w, dy, z, "silu"), ("d_x", "d_w", "d_b")):
            ref.check("%s %s" % (what, dtype), g, v, e)


def test_linear_huge_fp32():
    """Values past the largest bf16 and products that only just fit."""
    b, new = _b(), _gen(9)
    x, w = new(80, 64), new(70, 64)
    x[:, 5] = 3.4e38
    w[:, 5] = w[:, 5] * 1e-3
    y = b.corr_linear(x, w)
    wy, _, ey, _ = ref.linear(x, w, None, "none", None)
    ref.check("huge", y, wy, ey)


def test_linear_workspaces_streams_and_graphs():
    b, new = _b(), _gen(21)
    M, N, K = 300, 40, 4100
    x, w, bias, res = new(M, K, dtype=BF16), new(N, K, sigma=0.02, dtype=BF16), new(N), new(M, N, dtype=BF16)
    need = b.corr_linear_workspace_bytes(BF16, M, N, K)
    assert need > 0
    want = b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_GELU, residual=res)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    assert torch.equal(b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_GELU, residual=res, workspace=ws), want)
    with pytest.raises(ValueError):
        b.corr_linear(x, w, workspace=ws[:need - 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_GELU, residual=res)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    # a captured forward and backward, replayed between eager calls on changing inputs
    dy = new(M, N, dtype=BF16)
    z = torch.empty_like(res)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gy = b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_GELU, residual=res, preact=z)
        grads = b.corr_linear_backward(x, w, dy, preact=z, act=b.CORR_ACT_GELU)
    for k in range(4):
        x.copy_(new(M, K, dtype=BF16))
        dy.copy_(new(M, N, dtype=BF16))
        graph.replay()
        torch.cuda.synchronize()
        ez = torch.empty_like(z)
        ey = b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_GELU, residual=res, preact=ez)
        eg = b.corr_linear_backward(x, w, dy, preact=ez, act=b.CORR_ACT_GELU)
        assert torch.equal(gy, ey) and torch.equal(z, ez) and all(torch.equal(p, q) for p, q in zip(grads, eg)), k


# ---------------------------------------------------------------------------------------------------------------- norms

MIXES = [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16)]
# rows of every kernel, whole and odd: lanes of a row, one wave, several, sums kept in memory
COLS = [1, 5, 16, 63, 64, 136, 255, 256, 324, 512, 1000, 1024, 1027, 2048, 4096, 5000, 8191, 8192, 8200, 16384]
FORMS = [("none", "rms", None, False, 1.0), ("rms", "rms", "sigmoid", True, 1.0), ("layer", "layer", "silu", True, 2.5),
         ("rms", "none", "none", False, 1.0), ("none", "layer", "gelu", True, 1.0), ("layer", "rms", None, True, 0.5)]


def _case(S, T, rows, C, form, seed):
    post, pre, gate, scale, alpha = form
    new = _gen(seed)
    h = new(rows, C, sigma=2.0, mean=0.3, dtype=S)
    y = new(rows, C, sigma=0.7, mean=-0.2, dtype=T)
    vec = lambda mean, there: new(C, sigma=0.2, mean=mean) if there else None  # noqa: E731
    kw = dict(y=y, gate=new(rows, C, dtype=T) if gate else None, scale=vec(0.5, scale), h_scale=alpha,
              post_weight=vec(1.0, post != "none"), post_bias=vec(0.0, post == "layer"),
              pre_weight=vec(1.0, pre != "none"), pre_bias=vec(0.0, pre == "layer"))
    r = ref.Norm(h, y, kw["gate"], gate or "none", kw["scale"], alpha, post, kw["post_weight"], kw["post_bias"], pre, kw["pre_weight"],
                 kw["pre_bias"], 1e-5, T)
    kw.update(post=_norm(post), pre=_norm(pre), gate_act=_act(gate or "none"), eps=1e-5)
    return new, h, kw, r


@pytest.mark.parametrize("S,T", MIXES)
@pytest.mark.parametrize("C", COLS)
def test_norm_and_gradient(C, S, T):
    b = _b()
    form = FORMS[(COLS.index(C) + MIXES.index((S, T))) % len(FORMS)]
    for rows in (1, 37):
        new, h, kw, r = _case(S, T, rows, C, form, C + rows)
        t, n = b.corr_residual_norm(h, **kw)
        for g, (v, e), what in zip((t, n), r.forward(), ("h_out", "n_out")):
            ref.check("%s C=%d rows=%d %s" % (what, C, rows, form), g, v, e)
        assert t.dtype == S and (n is None or n.dtype == T)
        dh, dn = new(rows, C, dtype=S), new(rows, C, dtype=T) if form[1] != "none" else None
        got = b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw)
        for name, g, want in zip(got._fields, got, r.backward(dh, dn)):
            assert (g is None) == (want is None), name
            if g is not None:
                ref.check("%s C=%d rows=%d %s" % (name, C, rows, form), g, *want)
        again = b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw)
        assert all(p is q or torch.equal(p, q) for p, q in zip(got, again)), "two calls differ"


@pytest.mark.parametrize("S,T", [(F32, F32), (BF16, BF16), (F32, F16)])
@pytest.mark.parametrize("form", FORMS)
def test_norm_forms(form, S, T):
    """Every form on many rows (each thread has several), one of the two gradients absent in turn."""
    b, rows, C = _b(), 5003, 96
    new, h, kw, r = _case(S, T, rows, C, form, 5)
    for g, (v, e), what in zip(b.corr_residual_norm(h, **kw), r.forward(), ("h_out", "n_out")):
        ref.check("%s %s" % (what, form), g, v, e)
    dh, dn = new(rows, C, dtype=S), new(rows, C, dtype=T)
    for p, q in ((dh, dn), (None, dn), (dh, None)):
        if form[1] == "none":
            if p is None:
                continue
            q = None
        got = b.corr_residual_norm_backward(h, d_h_out=p, d_n_out=q, **kw)
        for i, (name, g, want) in enumerate(zip(got._fields, got, r.backward(p, q))):
            if g is not None:
                ref.check("%s %s" % (name, form), g, *want)
                # sums over 5003 rows of terms that are some EPS off, in random directions: far below the bounds' sums of magnitudes
                if i >= 3 and float(want[0].norm()):
                    assert float((g.double().cpu() - want[0]).norm() / want[0].norm()) < 1e-5, name


def test_norm_alone_and_wide_rows_without_their_gradient():
    """No block: the norm of h.  Rows whose column sums lie in memory, where d_n_out is absent."""
    b = _b()
    for S, T, C in ((F32, F32, 256), (F32, BF16, 33), (BF16, BF16, 9000)):
        new = _gen(C)
        h, w2, b2 = new(19, C, dtype=S), new(C, mean=1.0), new(C)
        r = ref.Norm(h, None, None, "none", None, 1.0, "none", None, None, "layer", w2, b2, 1e-5, T)
        t, n = b.corr_residual_norm(h, pre=b.CORR_NORM_LAYER, pre_weight=w2, pre_bias=b2, dtype=T)
        assert t is h
        ref.check("n", n, *r.forward()[0])
        dh, dn = new(19, C, dtype=S), new(19, C, dtype=T)
        for p in (dh, None):
            got = b.corr_residual_norm_backward(h, pre=b.CORR_NORM_LAYER, pre_weight=w2, pre_bias=b2, d_h_out=p, d_n_out=dn)
            want = r.backward(p, dn)
            for i in (0, 6, 7):
                ref.check(got._fields[i], got[i], *want[i])
    new, h, kw, r = _case(F32, BF16, 7, 9000, FORMS[2], 1)
    dh = new(7, 9000)
    got = b.corr_residual_norm_backward(h, d_h_out=dh, **kw)
    for name, g, want in zip(got._fields, got, r.backward(dh, None)):
        ref.check(name, g, *want)
    assert (got.d_pre_weight == 0).all() and (got.d_pre_bias == 0).all()


@pytest.mark.parametrize("C,ld", [(64, 80), (64, 67), (300, 301)])
def test_norm_strides_in_place_and_guards(C, ld):
    b = _b()
    new, _, kw, _ = _case(BF16, BF16, 21, C, FORMS[1], 2)
    wide = [new(21, ld, dtype=BF16) for _ in range(3)]
    h, y, gate = (t[:, :C] for t in wide)
    kw.update(y=y, gate=gate)
    r = ref.Norm(h, y, gate, "sigmoid", kw["scale"], 1.0, "rms", kw["post_weight"], None, "rms", kw["pre_weight"], None, 1e-5, BF16)
    buf = torch.full((23, C), 7.0, dtype=BF16, device="cuda")
    t, n = b.corr_residual_norm(h, n_out=buf[1:22], **kw)
    (wt, et), (wn, en) = r.forward()
    ref.check("h_out", t, wt, et)
    ref.check("n_out", n, wn, en)
    assert (buf[0] == 7).all() and (buf[22] == 7).all()
    acc = h.contiguous()
    b.corr_residual_norm(acc, h_out=acc, **kw)
    assert torch.equal(acc, t)
    dh, dn = new(21, C, dtype=BF16), new(21, C, dtype=BF16)
    got = b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw)
    for name, g, want in zip(got._fields, got, r.backward(dh, dn)):
        if g is not None:
            ref.check(name, g, *want)


@pytest.mark.parametrize("C", [8193, 8705, 9001])
def test_norm_sums_in_memory_of_ragged_rows(C):
    """More rows than workgroups, rows that end in a piece whose other columns belong to the next wave's neighbour or to another piece."""
    b, rows = _b(), 1100
    new, h, kw, r = _case(F32, F32, rows, C, FORMS[2], C)
    dh, dn = new(rows, C), new(rows, C)
    got = b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw)
    for i, want in enumerate(r.backward(dh, dn)):
        if i >= 3:
            ref.check("%s C=%d" % (got._fields[i], C), got[i], *want)
            rel = float((got[i].double().cpu() - want[0]).norm() / want[0].norm())
            assert rel < 1e-5, (got._fields[i], rel)     # one of 1100 rows counted twice is 1e-3


@pytest.mark.parametrize("C", [129, 516, 1027, 2049, 4100, 8191, 8705])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_in_place_ragged(C, dtype):
    """In place with rows that several waves share and that end inside a piece: as out of place, bit for bit."""
    b, rows = _b(), 900
    new = _gen(C)
    h, y, w = new(rows, C, dtype=dtype), new(rows, C, dtype=dtype), new(C, mean=1.0)
    t, n = b.corr_residual_norm(h, y=y, pre_weight=w)
    acc = h.clone()
    _, n2 = b.corr_residual_norm(acc, y=y, pre_weight=w, h_out=acc)
    assert torch.equal(acc, t) and torch.equal(n, n2)
    assert torch.equal(t, (h.float() + y.float()).to(dtype))


def test_norm_edges():
    """Rows of zeros (eps alone), of one value (no spread), very large and very small ones; a NaN stays in its row; no rows."""
    b = _b()
    h = torch.randn(6, 128).cuda()
    h[0], h[1], h[2], h[3] = 0.0, 3.0, h[2] * 1e15, h[3] * 1e-15
    for kind in ("rms", "layer"):
        r = ref.Norm(h, None, None, "none", None, 1.0, "none", None, None, kind, None, None, 1e-5, F32)
        ref.check(kind, b.corr_residual_norm(h, pre=_norm(kind))[1], *r.forward()[0])
    bad = h.clone()
    bad[4, 7] = float("nan")
    n = b.corr_residual_norm(bad, pre=b.CORR_NORM_RMS)[1]
    assert torch.isnan(n[4]).all() and torch.equal(n[[0, 1, 2, 3, 5]], b.corr_residual_norm(h, pre=b.CORR_NORM_RMS)[1][[0, 1, 2, 3, 5]])
    e, w = torch.empty(0, 128).cuda(), torch.ones(128).cuda()
    t, n = b.corr_residual_norm(e, y=e, scale=w, pre_weight=w)
    assert t.shape == n.shape == (0, 128)
    g = b.corr_residual_norm_backward(e, y=e, scale=w, pre_weight=w, d_h_out=e, d_n_out=e)
    assert (g.d_scale == 0).all() and (g.d_pre_weight == 0).all() and g.d_h.shape == (0, 128)


def test_norm_streams_and_graphs():
    b, rows, C = _b(), 300, 256
    new, h, kw, _ = _case(F32, BF16, rows, C, FORMS[2], 8)
    dh, dn = new(rows, C), new(rows, C, dtype=BF16)
    want = b.corr_residual_norm(h, **kw) + tuple(b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw))
    need = b.corr_residual_norm_backward_workspace_bytes(rows, C)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = b.corr_residual_norm(h, **kw) + tuple(b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, workspace=ws, **kw))
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b.corr_residual_norm(h, **kw) + tuple(b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw))
    for _ in range(4):
        h.copy_(new(rows, C))
        dn.copy_(new(rows, C, dtype=BF16))
        graph.replay()
        torch.cuda.synchronize()
        want = b.corr_residual_norm(h, **kw) + tuple(b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw))
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_offsets_past_32_bits():
    """More than 2^31 elements and 2^32 bytes: the first and the last rows, forward and gradients (whose other rows' d_out is zero)."""
    b = _b()
    M, K, N = (1 << 31) // 324 + 4001, 324, 16
    x = torch.zeros(M, K, dtype=BF16, device="cuda")
    some = torch.cat([torch.arange(40), torch.arange(M - 300, M)]).cuda()
    new = _gen(2)
    x[some] = new(340, K, dtype=BF16)
    w = new(N, K, sigma=0.1, dtype=BF16)
    y = b.corr_linear(x, w)
    wy, _, ey, _ = ref.linear(x[some], w, None, "none", None)
    ref.check("y", y[some], wy, ey)
    assert (y[40:50] == 0).all()
    dy = torch.zeros(M, N, dtype=BF16, device="cuda")
    dy[some] = new(340, N, dtype=BF16)
    d_x, d_w, d_b = b.corr_linear_backward(x, w, dy)
    for g, (v, e), what in zip((d_x[some], d_w, d_b), ref.linear_backward(x[some], w, dy[some], None, "none"), ("d_x", "d_w", "d_b")):
        ref.check(what, g, v, e)
    assert (d_x[100] == 0).all()
    del y, d_x, dy
    n = b.corr_residual_norm(x, pre=b.CORR_NORM_RMS)[1]
    r = ref.Norm(x[some], None, None, "none", None, 1.0, "none", None, None, "rms", None, None, 1e-5, BF16)
    ref.check("n", n[some], *r.forward()[0])
    g = b.corr_residual_norm_backward(x, pre=b.CORR_NORM_RMS, d_n_out=n)
    ref.check("d_h", g.d_h[some], *r.backward(None, n[some])[0])
    del x, n, g
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------------------ together

def test_gradients_against_differences():
    """fp32: the change of sum(c y) over a step of 2e is 2e <gradient, direction> up to e^2 and the calls' rounding (about 1e-6 of
    the sum of magnitudes over e)."""
    b, new, e = _b(), _gen(31), 2.0 ** -7
    M, N, K = 60, 40, 48
    x, w, bias, c = new(M, K), new(N, K, sigma=0.15), new(N), new(M, N)
    vx, vw, vb = new(M, K), new(N, K, sigma=0.15), new(N)

    def f(s):
        return float((b.corr_linear(x + s * vx, w + s * vw, bias=bias + s * vb, act=b.CORR_ACT_GELU) * c).double().sum())
    z = torch.empty(M, N).cuda()
    b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_GELU, preact=z)
    g = b.corr_linear_backward(x, w, c, preact=z, act=b.CORR_ACT_GELU)
    along = sum(float((p * q).double().sum()) for p, q in zip(g, (vx, vw, vb)))
    numeric = (f(e) - f(-e)) / (2 * e)
    # third derivatives: e^2 / 6 of a cubic form of unit directions over M N sums of K + 1 terms: below 1e-2 of the gradient's scale
    scale = sum(float((p * q).double().norm()) for p, q in zip(g, (vx, vw, vb)))
    print("linear: along %.6f, differences %.6f, scale %.3f" % (along, numeric, scale), flush=True)
    assert abs(along - numeric) <= 1e-2 * scale
    new, h, kw, _ = _case(F32, F32, 30, 64, FORMS[2], 4)
    dh, dn = new(30, 64), new(30, 64)
    keys = ("y", "gate", "scale", "post_weight", "post_bias", "pre_weight", "pre_bias")
    v = {k: new(*kw[k].shape, sigma=0.3) for k in keys}
    vh = new(30, 64)

    def f2(s):
        t, n = b.corr_residual_norm(h + s * vh, **{**kw, **{k: kw[k] + s * v[k] for k in keys}})
        return float((t * dh).double().sum() + (n * dn).double().sum())
    g = b.corr_residual_norm_backward(h, d_h_out=dh, d_n_out=dn, **kw)
    pairs = list(zip(g, [vh] + [v[k] for k in keys]))
    along = sum(float((p * q).double().sum()) for p, q in pairs)
    scale = sum(float((p * q).double().norm()) for p, q in pairs)
    numeric = (f2(e) - f2(-e)) / (2 * e)
    print("norm: along %.6f, differences %.6f, scale %.3f" % (along, numeric, scale), flush=True)
    assert abs(along - numeric) <= 1e-2 * scale


def test_lookup_block_and_back():
    """As a network uses them: lookup (channels last) -> projection -> norm -> widening product -> narrowing product -> gate, scale,
    residual and the next norm, and the gradient all the way to the feature maps, in fp32 against float64 (autograd and the oracle)."""
    import numpy as np
    from oracle import corr_oracle as oracle
    from paper_2505_16942_amd import synth
    b, C, B, H, W, L = _b(), 32, 1, 14, 18, 2
    f1, f2, c = synth.small_case(13, B, H, W, 64, flow_range=5.0)
    t1, t2, tc = (torch.from_numpy(a).cuda() for a in (f1, f2, c))
    pyr = b.corr_pyramid_build(t1, t2, L=L, reps=b.CORR_REP_F32)
    new, K = _gen(17), L * 81
    P = {"w0": new(C, K, sigma=K ** -0.5), "b0": new(C, sigma=0.1), "n1": new(C, sigma=0.1, mean=1.0), "w1": new(4 * C, C, sigma=C ** -0.5),
         "b1": new(4 * C, sigma=0.1), "w2": new(C, 4 * C, sigma=(4 * C) ** -0.5), "b2": new(C, sigma=0.1), "s": new(C, sigma=0.1, mean=0.5),
         "n2": new(C, sigma=0.1, mean=1.0), "c2": new(C, sigma=0.1)}
    corr = b.corr_sample(t1, pyr, tc, r=4, mode=b.CORR_MODE_ONDEMAND, layout=b.CORR_OUT_NHWC)
    z0, z1 = torch.empty(B, H, W, C).cuda(), torch.empty(B, H, W, 4 * C).cuda()
    h = b.corr_linear(corr, P["w0"], bias=P["b0"], act=b.CORR_ACT_RELU, preact=z0)
    _, n = b.corr_residual_norm(h, pre=b.CORR_NORM_RMS, pre_weight=P["n1"])
    u = b.corr_linear(n, P["w1"], bias=P["b1"], act=b.CORR_ACT_GELU, preact=z1)
    y = b.corr_linear(u, P["w2"], bias=P["b2"])
    kw = dict(y=y, scale=P["s"], pre=b.CORR_NORM_LAYER, pre_weight=P["n2"], pre_bias=P["c2"])
    t, n2 = b.corr_residual_norm(h, **kw)
    dt, dn = new(B, H, W, C), new(B, H, W, C)
    # back
    g = b.corr_residual_norm_backward(h, d_h_out=dt, d_n_out=dn, **kw)
    du, dw2, db2 = b.corr_linear_backward(u, P["w2"], g.d_y)
    d_n, dw1, db1 = b.corr_linear_backward(n, P["w1"], du, preact=z1, act=b.CORR_ACT_GELU)
    g1 = b.corr_residual_norm_backward(h, pre=b.CORR_NORM_RMS, pre_weight=P["n1"], d_h_out=g.d_h, d_n_out=d_n)
    d_corr, dw0, db0 = b.corr_linear_backward(corr, P["w0"], g1.d_h, preact=z0, act=b.CORR_ACT_RELU)
    d_f = b.corr_sample_backward(pyr, tc, d_corr.permute(0, 3, 1, 2).contiguous(), r=4)
    # float64
    x = corr.double().cpu().requires_grad_()
    Q = {k: v.double().cpu().requires_grad_() for k, v in P.items()}
    # the sign of the sum before the relu is the call's: a sum within rounding of zero has either slope
    mask = (z0 > 0).double().cpu()
    hq = (x @ Q["w0"].t() + Q["b0"]) * mask
    nq = hq / torch.sqrt((hq ** 2).mean(-1, keepdim=True) + 1e-5) * Q["n1"]
    yq = ref.act("gelu", nq @ Q["w1"].t() + Q["b1"]) @ Q["w2"].t() + Q["b2"]
    tq = hq + Q["s"] * yq
    dev = tq - tq.mean(-1, keepdim=True)
    oq = dev / torch.sqrt((dev ** 2).mean(-1, keepdim=True) + 1e-5) * Q["n2"] + Q["c2"]
    ((tq * dt.double().cpu()).sum() + (oq * dn.double().cpu()).sum()).backward()
    got = {"x": d_corr, "w0": dw0, "b0": db0, "n1": g1.d_pre_weight, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2, "s": g.d_scale,
           "n2": g.d_pre_weight, "c2": g.d_pre_bias}
    # ten fp32 steps, each within a few EPS sqrt(terms) of its own scale: 1e-5 in the 2-norm leaves a factor of ten, a lost term does not
    for name, value in [("t", (t, tq)), ("n", (n2, oq))] + [(k, (v, (x if k == "x" else Q[k]).grad)) for k, v in got.items()]:
        p, q = value[0].double().cpu().reshape(value[1].shape), value[1].detach()
        rel = float((p - q).norm() / q.norm())
        print("%s: %.2e" % (name, rel), flush=True)
        assert rel < 1e-5, name
    want = oracle.backward(f1, f2, c, x.grad.permute(0, 3, 1, 2).contiguous().numpy().astype(np.float32), L=L, r=4)
    for p, q in zip(d_f, want):
        rel = float(np.linalg.norm(p.cpu().numpy().astype(np.float64) - q) / np.linalg.norm(q))
        print("features: %.2e" % rel, flush=True)
        assert rel < 1e-5
    pyr.destroy()
