"""The fp16 gradient of a product with an activation: dz = d_y act'(z) has no place in one fp16 value.  A rounding of its own would make the
results' error sqrt 2 times that of their rounding, and d_y of 1e-5, which fp16 still holds to 1 in 170, times a slope of 1/10 would keep 1 in 17.

Against float64, rounded to fp16 once: an fp32 sum that is off by e (relative to the results' size, 1e-6 here) gives another
value than the nearest where the exact one lies within e of a border: of values as large as the rest 2 e / 2^-11 = 0.4 %, of smaller ones
more (their steps are finer), together about 1 %.  5 % is allowed; a rounding of dz changes a third of them and more.
"""
import pytest

import rows_reference as ref
from test_rows_tiles import DW, DX, FORMS, _sizes

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F16 = torch.float16


def _b():
    from paper_2505_16942_amd import binding
    return binding


def _case(M, N, K, sigma, name, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    new = lambda *shape, sigma=1.0: (torch.randn(shape, generator=g) * sigma).half().cuda()  # noqa: E731
    return new(M, K), new(N, K), new(M, N, sigma=sigma), new(M, N), getattr(_b(), "CORR_ACT_" + name.upper())


def _exact_dz(dy, z, name):
    return dy.double().cpu() * ref.slope(name, z.double().cpu())


def _check(what, got, want):
    got, want = got.double().cpu(), want
    off = (got != want.half().double()).double().mean()
    worst = float(((got - want).abs() / (ref.rounded(want, F16) + 1e-5 * want.norm() / want.numel() ** 0.5)).max())
    print("%s: %.2f %% not the nearest, worst %.2f of its bound" % (what, 100 * off, worst), flush=True)
    # beside the rounding 1e-5 of the results' size: sums of up to 5002 terms in fp32, each a few EPS sqrt(terms) off
    assert off < 0.05 and worst <= 1.0, what


@pytest.mark.parametrize("sigma", [0.3, 1e-5])
@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu", "sigmoid"])
def test_small_and_ordinary_gradients(name, sigma):
    b = _b()
    x, w, dy, z, act = _case(1500, 200, 150, sigma, name, 5)
    d_x, d_w, d_b = b.corr_linear_backward(x, w, dy, preact=z, act=act)
    dz = _exact_dz(dy, z, name)
    _check("d_x %s %g" % (name, sigma), d_x, dz @ w.double().cpu())
    _check("d_w %s %g" % (name, sigma), d_w, dz.t() @ x.double().cpu())
    assert float((d_b.double().cpu() - dz.sum(0)).norm() / dz.sum(0).norm()) < 1e-5


@pytest.mark.parametrize("product", [DX, DW])
@pytest.mark.parametrize("tile,split,R,C,S", [(tile, split, R, C, S) for tile, split, _, R, C, S in FORMS])
def test_every_tile(tile, split, R, C, S, product):
    """The tiles of test_rows_tiles.py, where this gradient has kernels of its own."""
    b = _b()
    M, N, K = _sizes(product, R, C, S)
    x, w, dy, z, act = _case(M, N, K, 1e-4, "silu", R + product)
    got = b.corr_linear_backward(x, w, dy, preact=z, act=act, want_x=product == DX, want_w=product == DW, want_bias=False)[product - 1]
    some = (torch.arange(R) if R < 700 else torch.cat([torch.arange(140), torch.arange(R // 2, R // 2 + 130), torch.arange(R - 300, R)])).cuda()
    if product == DX:
        want = _exact_dz(dy[some], z[some], "silu") @ w.double().cpu()
    else:
        want = _exact_dz(dy[:, some], z[:, some], "silu").t() @ x.double().cpu()
    _check("%s %s" % (tile, "split" if split else "whole"), got[some], want)
    again = b.corr_linear_backward(x, w, dy, preact=z, act=act, want_x=product == DX, want_w=product == DW, want_bias=False)[product - 1]
    assert torch.equal(got, again)


@pytest.mark.parametrize("N,K", [(40, 70), (41, 71)])
def test_not_finite(N, K):
    """Infinities and NaN reach what they reach in the sum of whole values: an infinite weight gives infinities with their signs, not NaN from two
    parts of opposite signs; d_y at the end of fp16's range times a slope above one is still finite."""
    b, M = _b(), 90
    x, w, dy, z, act = _case(M, N, K, 0.3, "gelu", N)
    w[3, 5] = float("inf")
    dy[7, 2] = float("-inf")
    dy[9, 4] = float("nan")
    z[11, 6], dy[11], w[6, 9] = 1.5, 0.0, 0.5            # gelu's slope there is 1.128
    dy[11, 6] = 65504.0
    d_x, d_w, _ = b.corr_linear_backward(x, w, dy, preact=z, act=act)
    dz = _exact_dz(dy, z, "gelu")
    for got, want in ((d_x, dz @ w.double().cpu()), (d_w, dz.t() @ x.double().cpu())):
        got = got.double().cpu()
        want = want.half().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.isinf() * got.sign().nan_to_num(), want.isinf() * want.sign().nan_to_num())
    assert torch.isfinite(d_x[11, 9]) and abs(float(d_x[11, 9]) - 0.5 * float(dz[11, 6])) <= 32


def test_captured_and_on_another_stream():
    """Both parts lie in the call's own workspace: replays between eager calls on changing inputs, and a call on another stream, give its bits."""
    b = _b()
    x, w, dy, z, act = _case(700, 126, 243, 0.05, "silu", 8)
    call = lambda **kw: b.corr_linear_backward(x, w, dy, preact=z, act=act, **kw)  # noqa: E731
    want = call()
    ws = torch.full((b.corr_linear_backward_workspace_bytes(F16, act, 700, 126, 243),), 0xff, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for k in range(4):
        _, _, dy_k, z_k, _ = _case(700, 126, 243, 0.05, "silu", 20 + k)
        dy.copy_(dy_k)
        z.copy_(z_k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, call())), k
