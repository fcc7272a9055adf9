"""corr_gated_linear and its gradient on the GPU against float64: every kind of tile, types, activations, layouts, values that are not finite, graphs.
The bounds are derived in maps_reference.py."""
import itertools

import pytest

import maps_reference as ref
from rows_reference import ACTS

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)


def _b():
    from paper_2505_16942_amd import binding
    return binding


def _act(name):
    return getattr(_b(), "CORR_ACT_" + name.upper())


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return lambda *shape, sigma=1.0, mean=0.0, dtype=F32: (torch.randn(shape, generator=g) * sigma + mean).to(dtype).cuda()


# (M, N, K): one element; few rows with whole, short and odd rows; a tile and its neighbours; odd everything; long k over few tiles
SIZES = [(1, 1, 1), (1, 16, 32), (1, 300, 1000), (3, 5, 7), (16, 256, 324), (17, 33, 65), (32, 130, 512), (33, 64, 64), (64, 32, 324), (65, 63, 243),
         (129, 127, 81), (130, 500, 36), (300, 8, 1024), (257, 129, 1100), (700, 128, 130), (40, 24, 4099), (77, 1, 5), (2000, 1, 1), (32, 33, 2051)]
# sizes that reach every kind of tile, whole and split: test_maps_api holds them to theirs
TILES = {"few": (20, 40, 100), "64": (100, 70, 100), "64 split": (100, 40, 4100), "128": (2570, 1030, 420), "128 split": (1030, 515, 4100),
         "256": (4090, 2045, 370), "rows": (33100, 250, 72)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_gated_linear(size, dtype):
    m, (M, N, K) = _b(), size
    new = _gen(M * 7 + N * 3 + K)
    x, w = new(M, K, dtype=dtype), new(2 * N, K, sigma=K ** -0.5, dtype=dtype)
    name = ACTS[(M + N + K) % 6]
    bias = new(2 * N, sigma=0.3) if (M + K) % 3 else None
    z = torch.full((M, 2 * N), float("nan"), dtype=dtype, device="cuda")
    y = m.corr_gated_linear(x, w, bias=bias, act=_act(name), preact=z)
    wy, wz, ey, ez = ref.gated(x, w, bias, name)
    ref.check("y %s %s %s" % (size, dtype, name), y, wy, ey)
    ref.check("z", z, wz, ez)
    assert torch.equal(y, m.corr_gated_linear(x, w, bias=bias, act=_act(name))), "two calls differ"
    # the sums are corr_linear's, of the same operands
    ref.check("z of corr_linear", m.corr_linear(x, w, bias=bias), wz, ez)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", sorted(TILES))
def test_every_tile(kind, dtype):
    m, (M, N, K) = _b(), TILES[kind]
    new = _gen(len(kind))
    x, w, bias = new(M, K, dtype=dtype), new(2 * N, K, sigma=K ** -0.5, dtype=dtype), new(2 * N, sigma=0.3)
    z = torch.full((M, 2 * N), float("nan"), dtype=dtype, device="cuda")
    y = m.corr_gated_linear(x, w, bias=bias, act=m.CORR_ACT_SILU, preact=z)
    wy, wz, ey, ez = ref.gated(x, w, bias, "silu")
    ref.check("%s y" % kind, y, wy, ey)
    ref.check("%s z" % kind, z, wz, ez)


# many rows of a short k, whose rows stay in registers: one and more pieces of k, half a chunk of 32 columns, odd numbers of chunks, all of 256 k
SHORT = [(230000, 33, 8), (60100, 250, 72), (153000, 96, 256), (14500, 1000, 200), (115100, 128, 128)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", SHORT)
def test_many_rows_of_a_short_k(size, dtype):
    """Columns of a wider buffer as rows, results apart, an infinity in one row: that row's sums alone, and nothing beside the results."""
    m, (M, N, K) = _b(), size
    new = _gen(M + N + K)
    wide = torch.full((M, K + 16), float("nan"), dtype=dtype, device="cuda")
    x = wide[:, 8:8 + K]
    x.copy_(new(M, K, dtype=dtype))
    w = new(2 * N, K, sigma=K ** -0.5, dtype=dtype)
    name = ACTS[(M + N + K) % 6]
    for bias in (None, new(2 * N, sigma=0.3)):
        z = torch.full((M + 1, 2 * N), 7.0, dtype=dtype, device="cuda")
        out = torch.full((M + 1, N + 3), 7.0, dtype=dtype, device="cuda")
        y = m.corr_gated_linear(x, w, bias=bias, act=_act(name), out=out[:M, 1:N + 1], preact=z[:M])
        assert (z[M] == 7).all() and (out[M] == 7).all() and (out[:, 0] == 7).all() and (out[:, N + 1:] == 7).all()
        assert torch.equal(y, m.corr_gated_linear(x, w, bias=bias, act=_act(name))), "with and without a preact differ"
        wy, wz, ey, ez = ref.gated(x, w, bias, name)
        ref.check("y %s %s %s" % (size, dtype, name), y, wy, ey)
        ref.check("z", z[:M], wz, ez)
    clean = m.corr_gated_linear(x, w, act=m.CORR_ACT_SIGMOID)
    x[M - 2, K - 1] = float("inf")
    got = m.corr_gated_linear(x, w, act=m.CORR_ACT_NONE, preact=z[:M])
    assert not z[M - 2].isfinite().any() and not got[M - 2].isfinite().any()
    got = m.corr_gated_linear(x, w, act=m.CORR_ACT_SIGMOID)
    assert torch.equal(got[:M - 2], clean[:M - 2]) and torch.equal(got[M - 1], clean[M - 1])


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_many_rows_on_borders_of_four_bytes(dtype):
    """x, its rows and w begin on 4-byte borders that are none of 16; an odd stride is another way through: the same sums within their bounds."""
    m, new = _b(), _gen(11)
    M, N, K = 60000, 256, 120
    even = torch.full((M, K + 6), float("nan"), dtype=dtype, device="cuda")[:, 2:K + 2]
    odd = torch.full((M, K + 5), float("nan"), dtype=dtype, device="cuda")[:, 4:K + 4]
    even.copy_(new(M, K, dtype=dtype))
    odd.copy_(even)
    w = torch.empty(2 * N * K + 2, dtype=dtype, device="cuda")[2:].view(2 * N, K)
    w.copy_(new(2 * N, K, sigma=K ** -0.5, dtype=dtype))
    assert even.data_ptr() % 16 == 4 and w.data_ptr() % 16 == 4
    wy, _, ey, _ = ref.gated(even, w, None, "gelu_tanh")
    for x in (even, odd):
        ref.check("y", m.corr_gated_linear(x, w, act=m.CORR_ACT_GELU_TANH), wy, ey)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_gated_linear_backward(size, dtype):
    m, (M, N, K) = _b(), size
    new = _gen(M * 5 + N * 11 + K)
    x, w, dy = new(M, K, dtype=dtype), new(2 * N, K, sigma=K ** -0.5, dtype=dtype), new(M, N, sigma=0.3, dtype=dtype)
    name, z = ACTS[(M + N) % 6], new(M, 2 * N, dtype=dtype)
    got = m.corr_gated_linear_backward(x, w, dy, z, act=_act(name))
    for g, (v, e), what in zip(got, ref.gated_backward(x, w, dy, z, name), ("d_x", "d_w", "d_b")):
        ref.check("%s %s %s %s" % (what, size, dtype, name), g, v, e)
    again = m.corr_gated_linear_backward(x, w, dy, z, act=_act(name))
    assert all(torch.equal(p, q) for p, q in zip(got, again)), "two calls differ"
    for want in itertools.product((False, True), repeat=3):
        part = m.corr_gated_linear_backward(x, w, dy, z, act=_act(name), want_x=want[0], want_w=want[1], want_bias=want[2])
        for p, q, wanted in zip(part, got, want):
            assert (p is None) if not wanted else torch.equal(p, q)


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations_far_out(name, dtype):
    """Every activation and slope at sums from -90 to 90."""
    m = _b()
    x = torch.linspace(-90, 90, 400).reshape(-1, 1).to(dtype).cuda()
    w = torch.tensor([[1.0], [0.5]], dtype=dtype, device="cuda")
    z = torch.empty(400, 2, dtype=dtype, device="cuda")
    y = m.corr_gated_linear(x, w, act=_act(name), preact=z)
    wy, _, ey, _ = ref.gated(x, w, None, name)
    ref.check("%s %s" % (name, dtype), y, wy, ey)
    dy = torch.ones_like(y)
    for g, (v, e), what in zip(m.corr_gated_linear_backward(x, w, dy, z, act=_act(name)), ref.gated_backward(x, w, dy, z, name), ("d_x", "d_w", "d_b")):
        # fp16's d_w is up to 1.1e6: from 65520 = 65504 + half a step on the nearest value of the type is infinity
        far = v.abs() - e >= 65520 if g.dtype == F16 else torch.zeros_like(v, dtype=torch.bool)
        g = g.double().cpu()
        assert torch.equal(g[far], torch.copysign(torch.full_like(v[far], float("inf")), v[far]))
        ref.check(what, torch.where(far, 0.0, g), torch.where(far, 0.0, v), e)


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Rows apart on both sides, columns of one buffer, d_out apart: the same bits; what lies between rows stays."""
    m, new = _b(), _gen(3)
    M, N, K = 150, 44, 70
    wide = torch.full((M, 3 * K), float("nan"), dtype=dtype, device="cuda")
    x = wide[:, K:2 * K]
    x.copy_(new(M, K, dtype=dtype))
    w, b, dy = new(2 * N, K, sigma=0.1, dtype=dtype), new(2 * N), new(M, N, dtype=dtype)
    z = torch.empty(M, 2 * N, dtype=dtype, device="cuda")
    want = m.corr_gated_linear(x.contiguous(), w, bias=b, preact=z)
    out = torch.full((M, 2 * N + 1), 7.0, dtype=dtype, device="cuda")
    m.corr_gated_linear(x, w, bias=b, out=out[:, 1:N + 1])
    assert torch.equal(out[:, 1:N + 1], want) and (out[:, 0] == 7).all() and (out[:, N + 1:] == 7).all()
    grads = m.corr_gated_linear_backward(x.contiguous(), w, dy, z)
    apart = torch.full((M, N + 3), float("nan"), dtype=dtype, device="cuda")
    apart[:, 1:N + 1] = dy
    got = m.corr_gated_linear_backward(x, w, apart[:, 1:N + 1], z)
    assert all(torch.equal(p, q) for p, q in zip(grads, got))
    assert m.corr_gated_linear(x.reshape(3, 50, K), w, bias=b).shape == (3, 50, N)


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_not_finite(dtype):
    """An infinity or NaN reaches its own row's sums and no other."""
    m, new = _b(), _gen(4)
    for M in (20, 200):
        x, w = new(M, 100, dtype=dtype), new(80, 100, sigma=0.1, dtype=dtype)
        clean = m.corr_gated_linear(x, w, act=m.CORR_ACT_SIGMOID)
        for junk in (float("nan"), float("inf")):
            bad = x.clone()
            bad[17, 99] = junk
            z = torch.empty(M, 80, dtype=dtype, device="cuda")
            y = m.corr_gated_linear(bad, w, act=m.CORR_ACT_SIGMOID, preact=z)
            assert not z[17].isfinite().any()
            rest = torch.arange(M, device="cuda") != 17
            assert torch.equal(y[rest], clean[rest])


def test_half_gradients_keep_small_and_large_values():
    """fp16 dz in two parts: gradients of 1e-6, and products of 1e5 beyond fp16's own range."""
    m, new = _b(), _gen(5)
    M, N, K = 300, 40, 64
    x, w, z = new(M, K, dtype=F16), new(2 * N, K, sigma=0.02, dtype=F16), new(M, 2 * N, dtype=F16)
    for sigma, up in ((1e-6, 1.0), (3e-4, 1.0), (10.0, 1000.0)):
        dy, zz = new(M, N, sigma=sigma, dtype=F16), z.clone()
        zz[:, N:] = (zz[:, N:].float() * up).clamp(-2500, 2500).to(F16)
        dy = dy.clamp(-30, 30)
        xs = (x.float() * (1.0 if up == 1.0 else 1e-3)).to(F16)
        for g, (v, e), what in zip(m.corr_gated_linear_backward(xs, w, dy, zz), ref.gated_backward(xs, w, dy, zz, "silu"), ("d_x", "d_w", "d_b")):
            ref.check("%s %g" % (what, sigma), g, v, e)


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16])
def test_factors_near_the_largest(dtype):
    """A second half of 3.3e38 where gelu's slope is 1.13: their product alone has no place in the type, the small gradient's has."""
    m, new = _b(), _gen(10)
    M, N, K = 40, 24, 32
    x, w, z = new(M, K, dtype=dtype), new(2 * N, K, sigma=0.1, dtype=dtype), new(M, 2 * N, dtype=dtype)
    z[:, :N], z[:, N:] = 1.5, 3.3e38
    dy = new(M, N, sigma=1e-6, dtype=dtype)
    for g, (v, e), what in zip(m.corr_gated_linear_backward(x, w, dy, z, act=m.CORR_ACT_GELU), ref.gated_backward(x, w, dy, z, "gelu"), ("d_x", "d_w", "d_b")):
        ref.check(what, g, v, e)


@pytest.mark.parametrize("name", ["none", "relu", "silu"])
def test_two_parts_of_the_largest_gradients(name):
    """bf16 dz in two parts up to 3.3e38: the second part is there also where 2048 times it has no place in the type."""
    m, new = _b(), _gen(12)
    M, N, K = 40, 24, 32
    x, w = new(M, K, sigma=1e-3, dtype=BF16), new(2 * N, K, sigma=1e-3, dtype=BF16)
    z = (torch.rand(M, 2 * N, generator=torch.Generator().manual_seed(4)) / 2 + 0.5).to(BF16).cuda()
    for most in (1e36, 1e38, 3.3e38):
        dy = ((torch.rand(M, N, generator=torch.Generator().manual_seed(3)) * 2 - 1) * most).to(BF16).cuda()
        got = m.corr_gated_linear_backward(x, w, dy, z, act=_act(name), want_bias=False)
        for g, (v, e), what in zip(got, ref.gated_backward(x, w, dy, z, name), ("d_x", "d_w")):
            ref.check("%s %g" % (what, most), g, v, e)


def test_differences():
    """The gradient against differences of the forward call in fp32: what the quotient itself is off by is computed in float64."""
    m, new = _b(), _gen(6)
    x, w, b, v = new(40, 30), new(24, 30, sigma=0.2), new(24), new(40, 12)
    z = torch.empty(40, 24, device="cuda")
    m.corr_gated_linear(x, w, bias=b, act=m.CORR_ACT_GELU, preact=z)
    grads = m.corr_gated_linear_backward(x, w, v, z, act=m.CORR_ACT_GELU)
    exact_z = ref.gated(x, w, b, "gelu")[1]
    h = 2.0 ** -6
    for i, t in enumerate((x, w, b)):
        step = new(*t.shape)
        sides, exact, noise = [], [], 0.0
        for sign in (1.0, -1.0):
            args = [x, w, b]
            args[i] = t + sign * h * step
            sides.append((m.corr_gated_linear(args[0], args[1], bias=args[2], act=m.CORR_ACT_GELU).double() * v.double()).sum().item())
            wy, _, ey, _ = ref.gated(*args, "gelu")
            exact.append((wy * v.double().cpu()).sum().item())
            noise += (ey * v.double().cpu().abs()).sum().item()
        along, e = ref.gated_backward(x, w, v, exact_z, "gelu")[i]
        # the gradient was taken at the stored z, which is 2^-24 of itself off: as much again
        e = e + 2.0 ** -20 * along.abs().max()
        true = (along * step.double().cpu()).sum().item()
        got = (grads[i].double() * step.double()).sum().item()
        truncation = abs((exact[0] - exact[1]) / (2 * h) - true)
        assert abs((sides[0] - sides[1]) / (2 * h) - got) <= truncation + noise / (2 * h) + (e * step.double().cpu().abs()).sum().item()
        assert truncation < 0.05 * abs(true) + 0.05


@pytest.mark.parametrize("dtype", TYPES)
def test_graphs(dtype):
    m = _b()
    M, N, K = 90, 40, 4100
    x, w, dy = _gen(7)(M, K, dtype=dtype), _gen(8)(2 * N, K, sigma=0.02, dtype=dtype), _gen(9)(M, N, dtype=dtype)
    y, z = torch.empty(M, N, dtype=dtype, device="cuda"), torch.empty(M, 2 * N, dtype=dtype, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(2 * N, device="cuda")
    wf = torch.empty(m.corr_gated_linear_workspace_bytes(dtype, M, N, K), dtype=torch.uint8, device="cuda")
    wb = torch.empty(m.corr_gated_linear_backward_workspace_bytes(dtype, M, N, K), dtype=torch.uint8, device="cuda")
    assert wf.numel() and wb.numel()

    def step():
        m.corr_gated_linear(x, w, out=y, preact=z, workspace=wf)
        m.corr_gated_linear_backward(x, w, dy, z, d_x=dx, d_w=dw, d_bias=db, workspace=wb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        x.copy_(_gen(70 + turn)(M, K, dtype=dtype))
        zz = torch.empty_like(z)
        want = m.corr_gated_linear(x, w, preact=zz)
        grads = m.corr_gated_linear_backward(x, w, dy, zz)
        for t in (y, z, dx, dw, db, wf, wb):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(z, zz) and all(torch.equal(p, q) for p, q in zip((dx, dw, db), grads)), turn


def test_nothing_to_do():
    m = _b()
    x, w = torch.empty(0, 16, device="cuda"), torch.ones(8, 16, device="cuda")
    assert m.corr_gated_linear(x, w).shape == (0, 4)
    dx, dw, db = m.corr_gated_linear_backward(x, w, torch.empty(0, 4, device="cuda"), torch.empty(0, 8, device="cuda"))
    assert dx.shape == (0, 16) and not dw.any() and not db.any()
