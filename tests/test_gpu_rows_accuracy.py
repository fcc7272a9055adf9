"""The row operators' activations and slopes, relative to their own values: on an exact sum (one term, weight 1), so that nothing else is
in the error.

EPS = 2^-24, one rounding; v_exp_f32 and v_rcp_f32 are off by one unit in the last place, 2 EPS.  Relative errors:
    e^-|z|            its argument is a product with a rounded constant: 2 |z| EPS, and 2 EPS
    sigmoid, silu     (2 |z| + 8) EPS: the exponential, 1 + e, the reciprocal, the product
    sigmoid's slope   (2 |z| + 16) EPS: e / (1 + e)^2, even in z
    gelu              the normal integral's tail: z^2 and two products with a rounded constant in the exponent, 1.5 z^2 EPS; a polynomial
                      of eight steps, a reciprocal and its denominator, three products: 32 EPS.  Of 1 - tail no more.
    gelu's slope      the same of the tail q and of |z| density, which have opposite signs below zero: relative to their sum
The product that carries the value adds 28 EPS (rows_reference.py's bound for a sum of one term).
"""
import math

import pytest

import rows_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)
EPS = ref.EPS


def _b():
    from paper_2505_16942_amd import binding
    return binding


def _values(dtype, most):
    """From -most to most, and normal ones; column of x."""
    g = torch.Generator()
    g.manual_seed(3)
    z = torch.cat([torch.linspace(-most, most, 4001), torch.randn(4000, generator=g) * 3])
    return z[z.abs() <= most].to(dtype).reshape(-1, 1).cuda()


def _forward(name, z):
    b = _b()
    return b.corr_linear(z, torch.ones(1, 1, dtype=z.dtype, device="cuda"), act=getattr(b, "CORR_ACT_" + name.upper()))


def _slope(name, z):
    b = _b()
    w = torch.ones(1, 1, dtype=z.dtype, device="cuda")
    return b.corr_linear_backward(z, w, torch.ones_like(z), preact=z, act=getattr(b, "CORR_ACT_" + name.upper()), want_w=False, want_bias=False)[0]


def _check(what, got, want, relative, dtype):
    # what lies below fp32's normal values may be taken as zero on the way
    bound = (relative + 28) * EPS * want.abs() + ref.rounded(want, dtype) + (1 + relative) * ref.TINY[F32]
    ref.check("%s %s" % (what, dtype), got, want, bound)


@pytest.mark.parametrize("dtype", TYPES)
def test_sigmoid_and_its_slope(dtype):
    """1 - sigmoid(z) cancels above zero; the slope is even and keeps its digits on both sides."""
    z = _values(dtype, 80.0)
    d = z.double().cpu()
    s = torch.sigmoid(d)
    _check("sigmoid", _forward("sigmoid", z), s, 2 * d.abs() + 8, dtype)
    _check("slope", _slope("sigmoid", z), s * torch.sigmoid(-d), 2 * d.abs() + 16, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_silu(dtype):
    z = _values(dtype, 80.0)
    d = z.double().cpu()
    _check("silu", _forward("silu", z), d * torch.sigmoid(d), 2 * d.abs() + 8, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_gelu_and_its_slope_keep_their_tails(dtype):
    z = _values(dtype, 12.0)
    d = z.double().cpu()
    tail = 0.5 * torch.erfc(d.abs() / math.sqrt(2.0))
    density = torch.exp(-0.5 * d * d) / math.sqrt(2 * math.pi)
    phi = torch.where(d < 0, tail, 1 - tail)
    per = 1.5 * d * d + 32
    _check("gelu", _forward("gelu", z), d * phi, per, dtype)
    want = phi + d * density
    apart = (phi + d.abs() * density) / want.abs().clamp_min(1e-30)
    _check("slope", _slope("gelu", z), want, (per + 28) * apart, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ref.ACTS[2:])
def test_huge_sums(name, dtype):
    """Far from zero an activation is its argument or zero (the sigmoid one or zero), its slope one or zero (the sigmoid's zero),
    also where squares and cubes on the way overflow."""
    big = [6e4] if dtype == F16 else [1e5, 1e15, 1e19, 1e20, 1e25, 3e38]
    z = torch.tensor(big + [-v for v in big]).to(dtype).reshape(-1, 1).cuda()
    up = (z > 0).double().cpu()
    want, slope = (up, 0 * up) if name == "sigmoid" else (z.double().cpu() * up, up)
    zero = torch.zeros_like(up)
    _check(name, _forward(name, z), want, zero, dtype)
    _check("slope of " + name, _slope(name, z), slope, zero, dtype)
