"""The row operators' refusals and host arithmetic: no device work.  Refused calls return before anything is enqueued, so made-up
addresses do."""
import os

import pytest

torch = pytest.importorskip("torch")


def _b():
    from paper_2505_16942_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("library not built (run __graft_entry__.build())")
    binding.load_library()
    return binding


# addresses far apart, one per matrix
X, W, BIAS, RES, PRE, Y, WS, DY, DX, DW, DB = (1 << 40 | (i << 34) for i in range(11))
MAX = 1 << 21


def _linear(b, **kw):
    a = dict(type=1, act=0, x=X, xs=64, w=W, bias=None, res=None, rs=0, pre=None, y=Y, ys=48, M=100, N=48, K=64, ws=WS, size=1 << 33)
    a.update(kw)
    return b.load_library().corr_linear(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), -1), (dict(type=-1), -1), (dict(act=6), -1), (dict(act=-1), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(y=None), -1),
    (dict(M=-1), -1), (dict(N=0), -1), (dict(K=0), -1), (dict(N=-4), -1), (dict(xs=63), -1), (dict(ys=47), -1), (dict(res=RES, rs=47), -1),
    (dict(M=(1 << 30) + 1), -2), (dict(N=MAX + 1, ys=MAX + 1), -2), (dict(K=MAX + 1, xs=MAX + 1), -2), (dict(xs=MAX + 1), -2),
    (dict(ys=MAX + 1), -2), (dict(res=RES, rs=MAX + 1), -2), (dict(M=1 << 30, N=128, ys=128), -2), (dict(M=1 << 30, K=128, xs=128), -2), (dict(N=1 << 19, ys=1 << 19, K=1 << 18, xs=1 << 18), -2),
    (dict(x=X + 2), -1), (dict(w=W + 2), -1), (dict(y=Y + 1), -1), (dict(bias=BIAS + 2), -1), (dict(pre=PRE + 1), -1), (dict(type=0, y=Y + 2), -1),
    (dict(res=RES + 1, rs=48), -1),
    # results that lie in what is read, or in each other; a residual that is nearly the result
    (dict(y=X), -1), (dict(y=W + 64), -1), (dict(pre=Y), -1), (dict(pre=X + 2 * 64 * 100 - 2), -1), (dict(bias=Y), -1),
    (dict(res=Y + 2, rs=48), -1), (dict(res=Y, rs=50), -1), (dict(res=PRE, rs=48, pre=PRE), -1),
    # a short, absent, crooked or overlapping workspace, where one is needed (a long k over few columns)
    (dict(K=4096, xs=4096, size=16), -1), (dict(K=4096, xs=4096, ws=None), -1), (dict(K=4096, xs=4096, ws=WS + 8), -1),
    (dict(K=4096, xs=4096, ws=X), -1), (dict(K=63, xs=63, size=0), -1), (dict(xs=65, ws=None), -1),
])
def test_linear_refusals(kw, status):
    assert _linear(_b(), **kw) == status


def test_no_rows_need_nothing():
    b = _b()
    assert _linear(b, M=0, x=None, w=None, y=None, ws=None, size=0) == 0
    assert b.corr_linear_workspace_bytes(torch.bfloat16, 0, 48, 64) == 0
    a = _norm(rows=0, h=None)
    assert b.load_library().corr_residual_norm(a, H_OUT, N_OUT, None) == 0


def _backward(b, **kw):
    a = dict(type=1, act=1, x=X, xs=64, w=W, pre=PRE, dy=DY, dys=48, dx=DX, dw=DW, db=DB, M=100, N=48, K=64, ws=WS, size=1 << 33)
    a.update(kw)
    return b.load_library().corr_linear_backward(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), -1), (dict(act=6), -1), (dict(dy=None), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(pre=None), -1), (dict(xs=63), -1),
    (dict(dys=47), -1), (dict(M=-1), -1), (dict(N=0), -1), (dict(K=0), -1), (dict(K=MAX + 1, xs=MAX + 1), -2), (dict(xs=MAX + 1), -2),
    (dict(dys=MAX + 1), -2), (dict(x=X + 2), -1), (dict(w=W + 2), -1), (dict(dy=DY + 2), -1), (dict(dx=DX + 1), -1), (dict(dw=DW + 1), -1),
    (dict(db=DB + 2), -1), (dict(pre=PRE + 1), -1), (dict(ws=None), -1), (dict(size=100), -1), (dict(ws=WS + 4), -1), (dict(dx=X), -1),
    (dict(dw=W), -1), (dict(dx=DY), -1), (dict(dw=DX), -1), (dict(db=DW), -1), (dict(ws=DY), -1), (dict(dx=PRE), -1),
])
def test_linear_backward_refusals(kw, status):
    assert _backward(_b(), **kw) == status


H, GATE, S1, P1, P2, P3, P4, H_OUT, N_OUT, DH, DN, D1, D2, D3, D4, D5, D6, D7, D8 = (1 << 41 | (i << 34) for i in range(19))


def _norm(**kw):
    from paper_2505_16942_amd import binding as b
    a = dict(stream_type=0, type=1, rows=10, cols=64, h=H, h_stride=64, y=Y, y_stride=64, gate=GATE, gate_stride=64, gate_act=5, scale=S1,
             h_scale=1.0, post=2, post_weight=P1, post_bias=P2, pre=1, pre_weight=P3, pre_bias=P4, eps=1e-5)
    a.update(kw)
    return b.residual_norm_args(*a.values())


NO_BLOCK = dict(y=None, y_stride=0, gate=None, gate_stride=0, scale=None, post=0, post_weight=None, post_bias=None)


@pytest.mark.parametrize("kw,outs,status", [
    (dict(stream_type=3), {}, -1), (dict(type=-1), {}, -1), (dict(stream_type=1, type=2), {}, -1), (dict(stream_type=1, type=0), {}, -1),
    (dict(gate_act=6), {}, -1), (dict(post=3), {}, -1), (dict(pre=-1), {}, -1), (dict(rows=-1), {}, -1), (dict(cols=0), {}, -1),
    (dict(eps=0.0), {}, -1), (dict(eps=-1.0), {}, -1), (dict(eps=float("nan")), {}, -1), (dict(h=None), {}, -1), (dict(h_stride=63), {}, -1),
    (dict(y_stride=63), {}, -1), (dict(gate_stride=63), {}, -1), (dict(cols=16385, h_stride=16385, y_stride=16385, gate_stride=16385), {}, -2),
    (dict(rows=(1 << 30) + 1), {}, -2), (dict(h_stride=(1 << 30) + 1), {}, -2), (dict(h=H + 2), {}, -1), (dict(y=Y + 1), {}, -1),
    (dict(scale=S1 + 2), {}, -1), (dict(post=0), {}, -1), (dict(pre=0), {"n_out": None}, -1),
    (dict(y=None), {}, -1), (dict(NO_BLOCK), {}, -1), (dict(NO_BLOCK, h_scale=2.0), {"h_out": None}, -1),
    (dict(NO_BLOCK, scale=S1), {"h_out": None}, -1), (dict(), {"n_out": None}, -1), (dict(), {"h_out": None, "n_out": None}, -1),
    (dict(), {"h_out": Y}, -1), (dict(), {"n_out": H}, -1), (dict(), {"n_out": H_OUT}, -1), (dict(), {"h_out": H + 4}, -1),
    (dict(h_stride=65), {"h_out": H}, -1), (dict(), {"n_out": S1}, -1), (dict(), {"n_out": N_OUT + 1}, -1),
])
def test_norm_refusals(kw, outs, status):
    b = _b()
    a, o = _norm(**kw), dict({"h_out": H_OUT, "n_out": N_OUT}, **outs)
    assert b.load_library().corr_residual_norm(a, o["h_out"], o["n_out"], None) == status


def test_norm_refuses_no_arguments():
    lib = _b().load_library()
    assert lib.corr_residual_norm(None, H_OUT, N_OUT, None) == -1
    assert lib.corr_residual_norm_backward(None, *[None] * 10, None, 0, None) == -1


@pytest.mark.parametrize("kw,outs,status", [
    (dict(), dict(dh=None, dn=None), -1), (dict(pre=0, pre_weight=None, pre_bias=None), dict(d7=None, d8=None), -1),
    (dict(NO_BLOCK), {}, -1), (dict(gate=None), {}, -1), (dict(scale=None), {}, -1), (dict(post_bias=None), {}, -1), (dict(pre_weight=None), {}, -1),
    (dict(), dict(ws=None), -1), (dict(), dict(size=64), -1), (dict(), dict(ws=WS + 8), -1), (dict(), dict(d1=DH), -1), (dict(), dict(d2=Y), -1),
    (dict(), dict(d2=D1), -1), (dict(), dict(d4=P1), -1), (dict(), dict(d4=D5), -1), (dict(), dict(ws=D1), -1), (dict(), dict(dn=DN + 1), -1),
    (dict(), dict(d4=D4 + 2), -1), (dict(eps=0.0), {}, -1),
])
def test_norm_backward_refusals(kw, outs, status):
    b = _b()
    o = dict(dh=DH, dn=DN, d1=D1, d2=D2, d3=D3, d4=D4, d5=D5, d6=D6, d7=D7, d8=D8, ws=WS, size=1 << 30)
    o.update(outs)
    a = _norm(**kw)
    assert b.load_library().corr_residual_norm_backward(a, *o.values(), None) == status


def test_workspace_sizes():
    """None for rows that fill the chip by themselves; a partial sum per split of a long k; copies of odd rows; the gradient's dz and
    column sums.  Zero for sizes that are refused."""
    b = _b()
    assert b.corr_linear_workspace_bytes(torch.bfloat16, 129600, 256, 324) == 0
    assert b.corr_linear_workspace_bytes(torch.bfloat16, 16, 256, 2047) == 0          # few rows are read as they are
    split = b.corr_linear_workspace_bytes(torch.bfloat16, 64, 64, 1 << 16)
    assert split > 0 and split % (64 * 64 * 4) == 0
    odd = b.corr_linear_workspace_bytes(torch.float16, 4096, 256, 243)
    assert odd >= 2 * 248 * (4096 + 256) and b.corr_linear_workspace_bytes(torch.float32, 129600, 256, 243) == 0
    assert b.corr_linear_workspace_bytes(torch.bfloat16, 4096, 256, 64, 65) >= 2 * 64 * 4096
    for t, e in ((torch.float32, 4), (torch.bfloat16, 2)):
        plain = b.corr_linear_backward_workspace_bytes(t, b.CORR_ACT_NONE, 4096, 256, 64)
        dz = b.corr_linear_backward_workspace_bytes(t, b.CORR_ACT_SILU, 4096, 256, 64)
        assert dz - plain == 4096 * 256 * e
    assert b.corr_linear_workspace_bytes(torch.bfloat16, 4, MAX + 1, 64) == 0
    assert b.corr_linear_backward_workspace_bytes(torch.bfloat16, 9, 4, 4, 64) == 0
    assert b.corr_residual_norm_backward_workspace_bytes(1, 256) == 5 * 256 * 4
    assert b.corr_residual_norm_backward_workspace_bytes(10 ** 6, 16384) < 512 * 5 * 16384 * 4 + 256
    assert b.corr_residual_norm_backward_workspace_bytes(4, 16385) == 0


def test_binding_refuses_host_tensors_and_other_types():
    b = _b()
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    for call in (lambda: b.corr_linear(x, w), lambda: b.corr_linear_backward(x, w, torch.zeros(4, 6)), lambda: b.corr_residual_norm(x),
                 lambda: b.corr_residual_norm_backward(x, d_h_out=x), lambda: b.corr_linear(None, w)):
        with pytest.raises(TypeError):
            call()


def test_rows_of_views():
    """Which views are rows: contiguous last dimension, one stride from row to row."""
    b = _b()
    t = torch.zeros(4, 6, 10)
    assert b._rows(t, "t") == (24, 10, 10) and b._rows(t[..., :7], "t") == (24, 7, 10) and b._rows(t[0, 0], "t") == (1, 10, 10)
    assert b._rows(t[:, 2], "t") == (4, 10, 60) and b._rows(t[:1, ::2], "t") == (3, 10, 20) and b._rows(t[:, :, :1], "t") == (24, 1, 10)
    assert b._rows(t[:0], "t") == (0, 10, 10)
    for bad in (t[..., ::2], t[:, :4], t.transpose(0, 1), torch.zeros(()), t.expand(3, 4, 6, 10)):
        with pytest.raises(ValueError):
            b._rows(bad, "t")
