"""Every tile of the row operators' products in each of the three layouts (y, d_x, d_w), whole and split, with ragged borders and a sum that ends
inside a step.  Which tile a size goes to is the library's choice, by rules that may change: the first test holds each case to
the tile that it is there for (host only), the second runs it."""
import os

import pytest

import rows_reference as ref

torch = pytest.importorskip("torch")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
Y, DX, DW = range(3)
HALVES = (BF16, F16)

# (tile, whether the sum is split, types, result's rows, its columns, the sum's length)
FORMS = [((256, 256), False, HALVES, 4090, 4100, 456),
         ((128, 256), False, HALVES, 33000, 300, 100),
         ((128, 128), False, HALVES + (F32,), 2600, 2100, 404),
         ((128, 128), True, HALVES + (F32,), 1002, 1030, 4204),
         ((64, 64), False, HALVES + (F32,), 330, 190, 100),
         ((64, 64), True, HALVES + (F32,), 100, 90, 5002)]
CASES = [(tile, split, t, product, R, C, S) for tile, split, types, R, C, S in FORMS for t in types for product in (Y, DX, DW)]
CASES += [((0, 16), False, t, Y, R, 300, 700) for t in HALVES + (F32,) for R in (9, 25)]


def _sizes(product, R, C, S):
    """(M, N, K) of a call whose y, d_x or d_w has R rows of C and sums of S terms."""
    return {Y: (R, C, S), DX: (R, S, C), DW: (S, R, C)}[product]


def _binding():
    from paper_2505_16942_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("library not built (run __graft_entry__.build())")
    return binding


@pytest.mark.parametrize("tile,split,dtype,product,R,C,S", CASES)
def test_the_case_reaches_its_tile(tile, split, dtype, product, R, C, S):
    rows, cols, splits = _binding().corr_debug_linear_tile(dtype, product, *_sizes(product, R, C, S))
    assert ((rows, cols), splits > 1) == (tile, split)
    if rows:
        assert R % rows and C % cols and S % (32 if dtype == F32 or tile == (128, 256) else 64), "borders and the sum's end lie inside"


def test_refusals():
    b = _binding()
    for bad in ((BF16, 3, 8, 8, 8), (BF16, -1, 8, 8, 8), (BF16, 0, 0, 8, 8), (BF16, 0, 8, 0, 8), (BF16, 0, 8, 8, (1 << 21) + 1)):
        with pytest.raises(b.CorrError):
            b.corr_debug_linear_tile(*bad)


def test_workspace_of_the_half_gradient():
    """fp16 with an activation that shapes dz holds it in two parts."""
    b = _binding()
    size = lambda act: b.corr_linear_backward_workspace_bytes(F16, act, 4096, 256, 64)  # noqa: E731
    assert size(b.CORR_ACT_RELU) - size(b.CORR_ACT_NONE) == 2 * 4096 * 256
    for act in (b.CORR_ACT_GELU, b.CORR_ACT_GELU_TANH, b.CORR_ACT_SILU, b.CORR_ACT_SIGMOID):
        assert size(act) - size(b.CORR_ACT_NONE) == 4 * 4096 * 256


@pytest.mark.gpu
@pytest.mark.parametrize("tile,split,dtype,product,R,C,S", CASES)
def test_tile(tile, split, dtype, product, R, C, S):
    """Some rows of the result, the first and last tiles' among them, against float64 (bounds in rows_reference.py)."""
    b = _binding()
    M, N, K = _sizes(product, R, C, S)
    g = torch.Generator()
    g.manual_seed(R + C + S + product)
    new = lambda *shape, sigma=1.0: (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()  # noqa: E731
    some = torch.arange(R) if R < 700 else torch.cat([torch.arange(140), torch.arange(R // 2, R // 2 + 130), torch.arange(R - 300, R)])
    some = some.cuda()
    x, w = new(M, K), new(N, K, sigma=K ** -0.5)
    if product == Y:
        bias, res = torch.randn(N, generator=g).cuda(), new(M, N)
        got = b.corr_linear(x, w, bias=bias, act=b.CORR_ACT_SILU, residual=res)
        want, _, bound, _ = ref.linear(x[some], w, bias, "silu", res[some])
    else:
        dy = new(M, N, sigma=0.3)
        only = dict(want_x=product == DX, want_w=product == DW, want_bias=False)
        got = b.corr_linear_backward(x, w, dy, **only)[product - 1]
        if product == DX:
            want, bound = ref.linear_backward(x[some], w, dy[some], None, "none")[0]
        else:
            want, bound = ref.linear_backward(x, w[some], dy[:, some], None, "none")[1]
    assert got.shape == (R, C)
    ref.check("%s %s product %d %s" % (tile, "split" if split else "whole", product, dtype), got[some], want, bound)
    if dtype == F32:
        # The bound's sum of magnitudes hides what is lost everywhere.  In the 2-norm roundings add up as a random walk, EPS / 2 times the root of
        # the sum's steps of the matrix cores (six for every 32 terms, by split: 7e-7 for 4204 terms, all in one); without one of
        # the six products it is 2e-3 (first part by second) or 3e-6 (third by first).
        rel = float((got[some].double().cpu() - want).norm() / want.norm())
        print("2-norm %.2e" % rel, flush=True)
        assert rel < 2e-6
