"""The refusals and host arithmetic of the operators on maps: no device work.  Refused calls return before anything is enqueued, so made-up
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


# addresses far apart, one per array
Q, K, V, OUT, LSE, LENGTHS, MASK, WS, D_OUT, DQ, DK, DV = (1 << 42 | (i << 36) for i in range(12))


def _attention(kw):
    from paper_2505_16942_amd import binding as b
    a = dict(type=1, B=2, Lq=300, Lk=500, H=4, HK=2, D=64, q=Q, q_item=300 * 256, q_row=256, q_head=64, k=K, k_item=500 * 128, k_row=128, k_head=64,
             v=V, v_item=500 * 128, v_row=128, v_head=64, scale=0.125, k_lengths=LENGTHS, key_mask=MASK)
    a.update({k: v for k, v in kw.items() if k in a})
    return b.attention_args(*a.values())


REFUSED = [
    (dict(type=3), -1), (dict(type=-1), -1), (dict(B=-1), -1), (dict(Lq=-1), -1), (dict(Lk=-1), -1), (dict(H=0), -1), (dict(HK=0), -1), (dict(H=3), -1),
    (dict(D=0), -1), (dict(D=-8), -1), (dict(D=12), -2), (dict(D=264), -2), (dict(H=130), -2), (dict(B=(1 << 20) + 1), -2), (dict(Lk=(1 << 30) + 1), -2),
    (dict(Lq=1 << 30), -2), (dict(Lq=1 << 29, B=4), -2), (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(q=Q + 2), -1),
    (dict(k=K + 2), -1), (dict(v=V + 1), -1), (dict(q_row=255), -1), (dict(k_head=63), -1), (dict(v_item=-2), -1), (dict(q_row=(1 << 21) + 2), -2),
    (dict(k_row=(1 << 21) + 2), -2), (dict(v_head=(1 << 21) + 2), -2), (dict(q_item=(1 << 40) + 2), -2), (dict(scale=0.0), -1), (dict(scale=-1.0), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(k_lengths=LENGTHS + 2), -1),
    (dict(B=1 << 20, H=1, HK=1, D=8, Lq=4096, Lk=8192), -2),          # more workgroups than a launch has
]


def _forward(b, **kw):
    o = dict(out=OUT, lse=LSE, ws=WS, size=1 << 33)
    o.update({k: v for k, v in kw.items() if k in o})
    return b.load_library().corr_attention(_attention(kw), o["out"], o["lse"], o["ws"], o["size"], None)


@pytest.mark.parametrize("kw,status", REFUSED + [
    (dict(out=None), -1), (dict(out=OUT + 1), -1), (dict(lse=LSE + 2), -1), (dict(Lk=50000, ws=None), -1), (dict(Lk=50000, size=64), -1),
    (dict(Lk=50000, ws=WS + 8), -1),
    (dict(out=Q), -1), (dict(out=K + 500 * 128 * 2), -1), (dict(out=V - 2), -1), (dict(lse=OUT), -1), (dict(Lk=50000, ws=OUT), -1), (dict(Lk=50000, ws=MASK), -1),
    (dict(out=LENGTHS), -1), (dict(lse=Q + 4), -1),
])
def test_attention_refusals(kw, status):
    assert _forward(_b(), **kw) == status


def _backward(b, **kw):
    o = dict(out=OUT, lse=LSE, d_out=D_OUT, dq=DQ, dk=DK, dv=DV, ws=WS, size=1 << 33)
    o.update({k: v for k, v in kw.items() if k in o})
    return b.load_library().corr_attention_backward(_attention(kw), *o.values(), None)


@pytest.mark.parametrize("kw,status", REFUSED + [
    (dict(out=None), -1), (dict(lse=None), -1), (dict(d_out=None), -1), (dict(d_out=D_OUT + 2), -1), (dict(dk=None), -1), (dict(dv=None), -1),
    (dict(dq=DQ + 1), -1), (dict(dk=DK + 1), -1), (dict(ws=None), -1), (dict(size=256), -1), (dict(ws=WS + 4), -1), (dict(dq=D_OUT), -1), (dict(dq=OUT), -1),
    (dict(dk=DV), -1), (dict(dk=K), -1), (dict(dv=Q), -1), (dict(dq=LSE), -1), (dict(ws=DQ), -1), (dict(ws=V), -1),
])
def test_attention_backward_refusals(kw, status):
    assert _backward(_b(), **kw) == status


def test_attention_without_work():
    b = _b()
    assert _forward(b, B=0, q=None, k=None, v=None, out=None, ws=None) == 0
    assert _forward(b, Lq=0, q=None, out=None, ws=None) == 0
    assert _backward(b, dq=None, dk=None, dv=None, ws=None) == 0
    assert _backward(b, B=0, out=None, lse=None, d_out=None, ws=None) == 0
    assert b.load_library().corr_attention(None, OUT, None, WS, 1 << 30, None) == -1
    for need in (b.corr_attention_workspace_bytes, b.corr_attention_backward_workspace_bytes):
        assert need(torch.bfloat16, 0, 5, 5, 1, 1, 64) == 0 and need(torch.bfloat16, 1, 0, 5, 1, 1, 64) == 0
        assert need(torch.bfloat16, 1, 5, 5, 1, 1, 20) == 0 and need(torch.bfloat16, 1, 5, 5, 3, 2, 64) == 0


def test_attention_workspace():
    """A few rows of many keys are split, and need room for the shares' sums; many rows need none; the gradient's holds two numbers a row at least."""
    b = _b()
    assert b.corr_attention_workspace_bytes(torch.bfloat16, 1, 1, 32768, 8, 2, 128) > 8 * 128 * 4
    assert b.corr_attention_workspace_bytes(torch.bfloat16, 1, 32400, 32400, 4, 4, 128) == 0
    assert b.corr_attention_backward_workspace_bytes(torch.bfloat16, 1, 32400, 32400, 8, 8, 64) < 32400 * 8 * 8 + 8 * 64 * 8 + 1024
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for Lq, Lk in ((1, 1), (1, 1 << 30), (1 << 30, 1), (100000, 100000)):
            assert b.corr_attention_backward_workspace_bytes(dtype, 1, Lq, Lk, 1, 1, 8) >= 8 * Lq


def test_binding_checks_before_the_library():
    b = _b()
    x = torch.zeros(1, 2, 2, 8)
    with pytest.raises((TypeError, ValueError)):
        b.corr_attention(x, x, x)                       # not on the GPU


X, Y, STATS, W, BIAS, DY, DX, DW, DB = (1 << 43 | (i << 36) for i in range(9))


def _norm(b, **kw):
    a = dict(type=1, act=1, x=X, xs=64, w=W, bias=BIAS, eps=1e-5, stats=STATS, y=Y, B=2, P=100, C=64, G=8, ws=WS, size=1 << 30)
    a.update(kw)
    return b.load_library().corr_group_norm(*a.values(), None)


NORM_REFUSED = [
    (dict(type=3), -1), (dict(act=6), -1), (dict(act=-1), -1), (dict(B=-1), -1), (dict(P=-1), -1), (dict(C=0), -1), (dict(G=0), -1), (dict(G=7), -1),
    (dict(G=128), -1), (dict(C=16392, xs=16392), -2), (dict(B=65536), -2), (dict(B=60000, C=256, xs=256), -2), (dict(P=1 << 30), -2),
    (dict(x=None), -1), (dict(xs=63), -1), (dict(xs=(1 << 21) + 1), -2), (dict(x=X + 1), -1), (dict(w=W + 2), -1), (dict(bias=BIAS + 1), -1),
    (dict(ws=None), -1), (dict(size=100), -1), (dict(ws=WS + 8), -1),
]


@pytest.mark.parametrize("kw,status", NORM_REFUSED + [
    (dict(eps=0.0), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(y=None), -1), (dict(y=Y + 1), -1), (dict(stats=STATS + 2), -1),
    (dict(y=X + 2), -1), (dict(y=X, xs=66), -1), (dict(y=W), -1), (dict(stats=Y), -1), (dict(ws=X), -1), (dict(ws=Y), -1), (dict(stats=X), -1),
])
def test_group_norm_refusals(kw, status):
    assert _norm(_b(), **kw) == status


@pytest.mark.parametrize("kw,status", NORM_REFUSED + [
    (dict(stats=None), -1), (dict(dy=None), -1), (dict(dys=63), -1), (dict(dys=(1 << 21) + 1), -2), (dict(dx=DX + 1), -1), (dict(dw=DW + 2), -1),
    (dict(db=DB + 1), -1), (dict(dx=X), -1), (dict(dx=DY), -1), (dict(dw=DX), -1), (dict(db=DW), -1), (dict(dw=STATS), -1), (dict(ws=DY), -1), (dict(db=W), -1),
])
def test_group_norm_backward_refusals(kw, status):
    b = _b()
    a = dict(type=1, act=1, x=X, xs=64, stats=STATS, w=W, bias=BIAS, dy=DY, dys=64, dx=DX, dw=DW, db=DB, B=2, P=100, C=64, G=8, ws=WS, size=1 << 30)
    a.update(kw)
    assert b.load_library().corr_group_norm_backward(*a.values(), None) == status


def test_group_norm_workspace():
    b = _b()
    for need in (b.corr_group_norm_workspace_bytes, b.corr_group_norm_backward_workspace_bytes):
        assert need(torch.float32, 0, 5, 8, 2) == 0 and need(torch.float32, 1, 0, 8, 2) == 0 and need(torch.float32, 1, 5, 8, 3) == 0
        for B, P, C, G in ((1, 1, 1, 1), (2, 518400, 256, 32), (65535, 3, 64, 2), (1, 1 << 30, 8, 8), (512, 16, 16384, 16384)):
            assert B * C * 8 <= need(torch.bfloat16, B, P, C, G) < (1 << 26) + 32 * B * C


Z = 1 << 44
MAX = 1 << 21


def _gated(b, **kw):
    a = dict(type=1, act=4, x=X, xs=64, w=W, bias=None, z=None, y=Y, ys=48, M=100, N=48, K=64, ws=WS, size=1 << 33)
    a.update(kw)
    return b.load_library().corr_gated_linear(*a.values(), None)


GATED_REFUSED = [
    (dict(type=3), -1), (dict(act=6), -1), (dict(M=-1), -1), (dict(N=0), -1), (dict(N=-1), -1), (dict(K=0), -1), (dict(M=(1 << 30) + 1), -2),
    (dict(N=MAX // 2 + 1), -2), (dict(N=1 << 62), -2), (dict(K=MAX + 1), -2), (dict(M=1 << 30, N=64), -2), (dict(xs=MAX + 1), -2), (dict(xs=63), -1),
    (dict(x=None), -1), (dict(w=None), -1), (dict(x=X + 2), -1), (dict(w=W + 2), -1),
]


@pytest.mark.parametrize("kw,status", GATED_REFUSED + [
    (dict(y=None), -1), (dict(ys=47), -1), (dict(ys=MAX + 1), -2), (dict(y=Y + 1), -1), (dict(bias=BIAS + 2), -1), (dict(z=Z + 1), -1), (dict(y=X), -1),
    (dict(y=W + 64), -1), (dict(z=Y), -1), (dict(z=W), -1), (dict(bias=Y), -1), (dict(K=4096, xs=4096, ws=None), -1), (dict(K=4096, xs=4096, size=16), -1),
    (dict(K=4096, xs=4096, ws=WS + 8), -1), (dict(K=63, xs=63, size=0), -1),
])
def test_gated_linear_refusals(kw, status):
    assert _gated(_b(), **kw) == status


@pytest.mark.parametrize("kw,status", GATED_REFUSED + [
    (dict(z=None), -1), (dict(z=Z + 1), -1), (dict(dy=None), -1), (dict(dy=DY + 1), -1), (dict(dys=47), -1), (dict(dys=MAX + 1), -2), (dict(dx=DX + 1), -1),
    (dict(dw=DW + 1), -1), (dict(db=DB + 2), -1), (dict(ws=None), -1), (dict(size=100), -1), (dict(ws=WS + 4), -1), (dict(dx=X), -1), (dict(dw=W), -1),
    (dict(dx=DY), -1), (dict(dw=DX), -1), (dict(db=DW), -1), (dict(ws=DY), -1), (dict(dx=Z), -1),
])
def test_gated_linear_backward_refusals(kw, status):
    b = _b()
    a = dict(type=1, act=4, x=X, xs=64, w=W, z=Z, dy=DY, dys=48, dx=DX, dw=DW, db=DB, M=100, N=48, K=64, ws=WS, size=1 << 33)
    a.update(kw)
    assert b.load_library().corr_gated_linear_backward(*a.values(), None) == status


def test_gated_tiles():
    """The sizes that the GPU tests use to reach every kind of tile do so."""
    b = _b()
    import test_gpu_gated_linear as t
    kinds = {"few": (0, 16), "64": (64, 64), "64 split": (64, 64), "128": (128, 128), "128 split": (128, 128), "256": (256, 256), "rows": (128, 256)}
    for dtype in t.TYPES:
        for kind, (M, N, K) in t.TILES.items():
            rows, cols, splits = b.corr_debug_linear_tile(dtype, 0, M, 2 * N, K)
            want = kinds[kind]
            if dtype == torch.float32 and kind in ("256", "rows"):
                want = (128, 128)
            assert (rows, cols) == want, (dtype, kind, rows, cols)
            assert ("split" in kind) == (splits > 1), (dtype, kind, splits)


def test_gated_tiles_of_a_short_k():
    """The sizes that are there for rows in registers go there; few rows or ones that leave XCDs idle, other lengths and fp32 go to the products' tiles."""
    b = _b()
    import test_gpu_gated_linear as t
    short = (128, 64, 1)
    for dtype in (torch.bfloat16, torch.float16):
        for size in t.SHORT + [(60000, 256, 120), (32400, 1024, 256), (129600, 512, 256)]:
            assert b.corr_debug_gated_tile(dtype, *size) == short, size
        for M, N, K in [(1, 114688, 256), (16, 1 << 20, 64), (33, 114688, 256), (128, 500000, 128), (1000, 14336, 256), (2500, 5760, 256), (9300, 1600, 256),
                        (32400, 1024, 264), (32400, 1024, 252)] + list(t.TILES.values()):
            tile = b.corr_debug_gated_tile(dtype, M, N, K)
            assert tile != short and tile == b.corr_debug_linear_tile(dtype, 0, M, 2 * N, K), (M, N, K)
    assert b.corr_debug_gated_tile(torch.float32, 32400, 1024, 256) == (128, 128, 1)
    for bad in ((torch.bfloat16, 0, 8, 8), (torch.bfloat16, 8, 0, 8), (torch.bfloat16, 8, 8, 0), (torch.bfloat16, 8, (1 << 20) + 1, 8)):
        with pytest.raises(b.CorrError):
            b.corr_debug_gated_tile(*bad)


def test_attention_scales():
    """scale log2 e has to be finite; without keys and rows the checks alone answer."""
    b = _b()
    for scale, status in ((2.0 ** 127, 0), (2.0 ** -149, 0), (1.8e38, -1), (3.4e38, -1), (-2.0 ** -149, -1)):
        assert _forward(b, B=0, q=None, k=None, v=None, out=None, ws=None, scale=scale) == status
        assert _backward(b, B=0, out=None, lse=None, d_out=None, ws=None, scale=scale) == status
