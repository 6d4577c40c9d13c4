"""What the entry points of the 4-bit products and of the mixture of experts refuse, on the host, before any launch."""
import ctypes

import pytest

import paper_2001_00532_amd as psk

torch = pytest.importorskip("torch")

ONE, NULL, ODD, BIG = ctypes.c_void_p(256), ctypes.c_void_p(0), ctypes.c_void_p(257), 1 << 30


def q4(**over):
    d = psk.psk_q4()
    d.count, d.rows, d.cols, d.group, d.scale_type = 1, 48, 100, 32, psk.PSK_BF16
    d.codes, d.scales, d.zeros = 256, 256, 256
    d.ld_codes, d.ld_scales, d.stride_codes, d.stride_scales = 64, 4, 64 * 48, 4 * 48
    for k, v in over.items():
        setattr(d, k, v)
    return d


def gemm(A=None, n=4, type=psk.PSK_BF16, X=ONE, ldx=100, Y=ONE, ldy=48, ws=ONE, have=BIG):
    A = q4() if A is None else A
    return psk.lib().psk_gemm_q4(ctypes.byref(A), n, type, X, ldx, Y, ldy, ws, have, NULL)


def test_gemm_q4_refuses():
    assert gemm(n=0) == 0 and gemm(q4(rows=0), ldy=0) == 0            # nothing to do: no launch
    assert psk.lib().psk_gemm_q4(None, 1, 1, ONE, 100, ONE, 48, ONE, BIG, NULL) == 1
    for over in (dict(codes=0), dict(scales=0)):
        assert gemm(q4(**over)) == 1, over
    assert gemm(X=NULL) == 1 and gemm(Y=NULL) == 1
    for over in (dict(rows=-1), dict(cols=-1), dict(cols=2 ** 28 + 1), dict(rows=2 ** 31), dict(group=0), dict(group=16), dict(group=96), dict(group=-32),
                 dict(ld_codes=48), dict(ld_scales=3), dict(count=2), dict(count=0), dict(count=-1)):
        assert gemm(q4(**over)) == 2, over
    assert gemm(n=-1) == 2 and gemm(n=psk.PSK_MAX_VECTORS + 1) == 2 and gemm(ldx=99) == 2 and gemm(ldy=47) == 2
    assert gemm(ws=NULL) == 4 and gemm(ws=ctypes.c_void_p(264)) == 4 and gemm(have=255) == 4
    assert gemm(type=3) == 5 and gemm(type=-1) == 5
    assert gemm(q4(scale_type=psk.PSK_F16)) == 5 and gemm(type=psk.PSK_F32) == 5 and gemm(q4(scale_type=3)) == 5
    for over in (dict(codes=264), dict(ld_codes=72), dict(scales=257)):
        assert gemm(q4(**over)) == 7, over
    assert gemm(q4(scale_type=psk.PSK_F32, scales=258)) == 7
    assert gemm(X=ODD) == 7 and gemm(Y=ODD) == 7
    assert psk.psk_gemm_q4_workspace_bytes(48, 100, 4, psk.PSK_F32) >= 256
    assert psk.psk_gemm_q4_workspace_bytes(-1, 100, 4, 0) == 0 and psk.psk_gemm_q4_workspace_bytes(48, 100, 4, 3) == 0
    assert psk.psk_gemm_q4_workspace_bytes(48, 100, psk.PSK_MAX_VECTORS + 1, 0) == 0


def route(n=4, dim=100, experts=10, top_k=3, score=0, type=psk.PSK_BF16, X=ONE, ldx=100, wtype=psk.PSK_BF16, W=ONE, ldw=100, bias=NULL, crd=ONE,
          vals=ONE, ws=ONE, have=BIG):
    return psk.lib().psk_moe_route(n, dim, experts, top_k, score, 1, 1.0, type, X, ldx, wtype, W, ldw, bias, crd, vals, ws, have, NULL)


def test_route_refuses():
    assert route(n=0) == 0
    for over in (dict(X=NULL), dict(W=NULL), dict(crd=NULL), dict(vals=NULL)):
        assert route(**over) == 1, over
    for over in (dict(n=-1), dict(n=psk.PSK_MAX_VECTORS + 1), dict(dim=0), dict(experts=0), dict(experts=psk.PSK_MOE_MAX_EXPERTS + 1), dict(top_k=0),
                 dict(top_k=psk.PSK_MOE_MAX_TOP_K + 1), dict(ldx=99), dict(ldw=99)):
        assert route(**over) == 2, over
    assert route(ws=NULL) == 4 and route(have=255) == 4 and route(ws=ODD) == 4
    assert route(have=psk.psk_moe_route_workspace_bytes(4, 10) - 1) == 4
    for over in (dict(score=2), dict(type=3), dict(wtype=psk.PSK_F16), dict(type=psk.PSK_F32)):
        assert route(**over) == 5, over
    for over in (dict(X=ODD), dict(W=ODD), dict(bias=ctypes.c_void_p(258)), dict(crd=ctypes.c_void_p(258)), dict(vals=ctypes.c_void_p(258))):
        assert route(**over) == 7, over
    assert psk.psk_moe_route_workspace_bytes(4, 1025) == 0 and psk.psk_moe_route_workspace_bytes(-1, 4) == 0
    assert psk.psk_moe_route_workspace_bytes(100, 64) >= 100 * 64 * 8


def layer(n=4, dim=100, inter=48, experts=10, top_k=3, act=0, type=psk.PSK_BF16, X=ONE, ldx=100, crd=ONE, vals=ONE, W1=ONE, W3=ONE, ld1=104,
          stride1=104 * 48, W2=ONE, ld2=48, stride2=4800, Y=ONE, ldy=100, ws=ONE, have=BIG):
    return psk.lib().psk_moe_experts(n, dim, inter, experts, top_k, act, type, X, ldx, crd, vals, W1, W3, ld1, stride1, W2, ld2, stride2, Y, ldy, ws, have, NULL)


def test_layer_refuses():
    assert layer(n=0) == 0
    for over in (dict(X=NULL), dict(crd=NULL), dict(vals=NULL), dict(W1=NULL), dict(W3=NULL), dict(W2=NULL), dict(Y=NULL)):
        assert layer(**over) == 1, over
    for over in (dict(n=-1), dict(n=psk.PSK_MAX_VECTORS + 1), dict(dim=0), dict(inter=0), dict(experts=0), dict(experts=1025), dict(top_k=0), dict(top_k=65),
                 dict(ldx=99), dict(ldy=99), dict(ld1=99), dict(ld2=47), dict(stride1=-8)):
        assert layer(**over) == 2, over
    assert layer(ws=NULL) == 4 and layer(have=psk.psk_moe_workspace_bytes(4, 100, 48, 10, 3) - 1) == 4
    for over in (dict(act=2), dict(type=psk.PSK_F32), dict(type=3)):
        assert layer(**over) == 5, over
    for over in (dict(X=ODD), dict(Y=ODD), dict(W1=ODD), dict(W3=ODD), dict(W2=ODD), dict(crd=ctypes.c_void_p(258))):
        assert layer(**over) == 7, over
    assert psk.psk_moe_workspace_bytes(4, 100, 0, 10, 3) == 0 and psk.psk_moe_workspace_bytes(4, 100, 48, 2000, 3) == 0
    # more tokens than one pair of launches takes need no more room
    assert psk.psk_moe_workspace_bytes(psk.PSK_MAX_VECTORS, 100, 48, 10, 8) == psk.psk_moe_workspace_bytes(4096, 100, 48, 10, 8)


def layer_q4(w1=None, w3=None, w2=None, n=4, top_k=3, act=0, type=psk.PSK_BF16, X=ONE, ldx=100, crd=ONE, vals=ONE, Y=ONE, ldy=100, ws=ONE, have=BIG):
    w1, w3, w2 = w1 or q4(count=10), w3 or q4(count=10), w2 or q4(count=10, rows=100, cols=48, ld_codes=32, ld_scales=2)
    return psk.lib().psk_moe_experts_q4(n, top_k, act, type, X, ldx, crd, vals, ctypes.byref(w1), ctypes.byref(w3), ctypes.byref(w2), Y, ldy, ws, have, NULL)


def test_layer_q4_refuses():
    assert layer_q4(n=0) == 0
    assert psk.lib().psk_moe_experts_q4(4, 3, 0, 2, ONE, 100, ONE, ONE, None, None, None, ONE, 100, ONE, BIG, NULL) == 1
    for over in (dict(X=NULL), dict(crd=NULL), dict(vals=NULL), dict(Y=NULL)):
        assert layer_q4(**over) == 1, over
    for over in (dict(w3=q4(count=9)), dict(w3=q4(count=10, rows=47)), dict(w3=q4(count=10, cols=99)), dict(w2=q4(count=10)), dict(w1=q4(count=0)),
                 dict(w1=q4(count=10, stride_codes=-16)), dict(w3=q4(count=10, group=64)), dict(ldx=99), dict(ldy=99), dict(top_k=0), dict(n=-1)):
        assert layer_q4(**over) == 2, over
    assert layer_q4(ws=NULL) == 4 and layer_q4(have=255) == 4
    assert layer_q4(w3=q4(count=10, scale_type=psk.PSK_F32)) == 5 and layer_q4(type=psk.PSK_F32) == 5 and layer_q4(act=7) == 5
    assert layer_q4(w1=q4(count=10, stride_codes=40)) == 7 and layer_q4(X=ODD) == 7


def test_largest_sizes():
    """One row or column more than a launch has threads for is refused, as many as it has are not (X = NULL is, after that)."""
    most = 2 ** 28 - 256
    big = dict(ld_codes=1 << 28, ld_scales=1 << 28, stride_codes=0, stride_scales=0)
    for rows, cols in ((most, 100), (48, most)):
        assert gemm(q4(rows=rows, cols=cols, **big), X=NULL, ldx=1 << 28, ldy=1 << 28, have=1 << 50) == 1
        assert psk.psk_gemm_q4_workspace_bytes(rows, cols, 5, psk.PSK_BF16) > 0 and psk.psk_moe_workspace_bytes(5, rows, cols, 3, 2) > 0
        assert layer(dim=rows, inter=cols, X=NULL, ldx=1 << 28, ldy=1 << 28, ld1=1 << 28, ld2=1 << 28, have=1 << 50) == 1
    for rows, cols in ((most + 1, 100), (48, most + 1), (2 ** 28, 100), (48, 2 ** 28)):
        assert gemm(q4(rows=rows, cols=cols, **big), X=NULL, ldx=1 << 28, ldy=1 << 28, have=1 << 50) == 2
        assert psk.psk_gemm_q4_workspace_bytes(rows, cols, 5, psk.PSK_BF16) == 0 and psk.psk_moe_workspace_bytes(5, rows, cols, 3, 2) == 0
        assert layer(dim=rows, inter=cols, X=NULL, ldx=1 << 28, ldy=1 << 28, ld1=1 << 28, ld2=1 << 28, have=1 << 50) == 2
        w = dict(count=10, **big)
        assert layer_q4(q4(rows=cols, cols=rows, **w), q4(rows=cols, cols=rows, **w), q4(rows=rows, cols=cols, **w), X=NULL, ldx=1 << 28, ldy=1 << 28) == 2
    assert route(dim=most, X=NULL, ldx=1 << 28, ldw=1 << 28) == 1 and route(dim=most + 1, X=NULL, ldx=1 << 28, ldw=1 << 28) == 2


def test_binding_refuses():
    """Shapes and types are checked before an address is asked for, host tensors when it is."""
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2)
    with pytest.raises(ValueError):
        psk.Q4(codes, scales, cols=64, group=48)
    with pytest.raises(ValueError):
        psk.Q4(codes, scales, cols=65, group=32)             # a row of codes too short
    with pytest.raises(ValueError):
        psk.Q4(codes, scales, cols=64, group=64)             # two scales per row where one is needed
    with pytest.raises(ValueError):
        psk.Q4(codes, scales, torch.zeros(8, 3, dtype=torch.uint8)[:, :2], cols=64, group=32)
    with pytest.raises(ValueError):
        psk.Q4(codes.int(), scales, cols=64, group=32)
    with pytest.raises(ValueError):
        psk.Q4(codes, scales, cols=64, group=32)             # on the host
    x, crd, vals = torch.zeros(3, 16).half(), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    w1, w2 = torch.zeros(4, 8, 16).half(), torch.zeros(4, 16, 8).half()
    for bad in (dict(crd=crd[:2]), dict(vals=vals[:, :1]), dict(W1=w1[:, :, :8]), dict(W2=w1), dict(Y=x[:, :8]), dict()):
        a = dict(X=x, crd=crd, vals=vals, W1=w1, W3=w1, W2=w2, Y=x)
        a.update(bad)
        with pytest.raises(ValueError):
            psk.psk_moe_experts(**a)
    with pytest.raises(ValueError):
        psk.psk_moe_route(x, torch.zeros(4, 16).half(), crd, vals, bias=torch.zeros(5))
    with pytest.raises(ValueError):
        psk.psk_moe_route(x.double(), torch.zeros(4, 16).double(), crd, vals)
