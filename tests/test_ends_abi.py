"""What the entry points of the products of 8-bit integers and of the embedding refuse, on the host, before any launch."""
import ctypes

import pytest

import paper_2001_00532_amd as psk

torch = pytest.importorskip("torch")

ONE, NULL, ODD, BIG = ctypes.c_void_p(256), ctypes.c_void_p(0), ctypes.c_void_p(257), 1 << 40
AT2, AT8 = ctypes.c_void_p(258), ctypes.c_void_p(264)


def i8(**over):
    d = psk.psk_i8()
    d.rows, d.cols, d.ld, d.codes, d.scales = 48, 100, 112, 256, 256
    for k, v in over.items():
        setattr(d, k, v)
    return d


def quant(n=4, cols=100, type=psk.PSK_BF16, X=ONE, ldx=100, codes=ONE, ldc=112, scales=ONE):
    return psk.lib().psk_quant_i8(n, cols, type, X, ldx, codes, ldc, scales, NULL)


def test_quant_refuses():
    assert quant(n=0) == 0
    for over in (dict(X=NULL), dict(codes=NULL), dict(scales=NULL)):
        assert quant(**over) == 1, over
    for over in (dict(n=-1), dict(n=2 ** 28), dict(cols=-1), dict(cols=psk.PSK_I8_MAX_COLS + 1, ldx=1 << 18, ldc=1 << 18), dict(ldx=99), dict(ldx=2 ** 31), dict(ldc=96),
                 dict(ldc=2 ** 23 + 16)):
        assert quant(**over) == 2, over
    assert quant(type=3) == 5 and quant(type=-1) == 5
    for over in (dict(X=ODD), dict(codes=AT8), dict(ldc=120), dict(scales=AT2), dict(type=psk.PSK_F32, X=AT2)):
        assert quant(**over) == 7, over


def gemm(A=None, n=4, X=ONE, ldx=112, scales=ONE, bias=NULL, type=psk.PSK_BF16, Y=ONE, ldy=48, ws=ONE, have=BIG):
    A = i8() if A is None else A
    return psk.lib().psk_gemm_i8(ctypes.byref(A), n, X, ldx, scales, bias, type, Y, ldy, ws, have, NULL)


def linear(A=None, n=4, type=psk.PSK_BF16, X=ONE, ldx=100, bias=NULL, Y=ONE, ldy=48, ws=ONE, have=BIG):
    A = i8() if A is None else A
    return psk.lib().psk_linear_i8(ctypes.byref(A), n, type, X, ldx, bias, Y, ldy, ws, have, NULL)


@pytest.mark.parametrize("call", [gemm, linear])
def test_products_refuse(call):
    assert call(n=0) == 0 and call(i8(rows=0), ldy=0) == 0
    for over in (dict(codes=0), dict(scales=0)):
        assert call(i8(**over)) == 1, over
    assert call(X=NULL) == 1 and call(Y=NULL) == 1
    for over in (dict(rows=-1), dict(rows=2 ** 28), dict(cols=-1), dict(cols=psk.PSK_I8_MAX_COLS + 1, ld=1 << 18), dict(ld=96), dict(ld=2 ** 23 + 16)):
        assert call(i8(**over)) == 2, over
    assert call(n=-1) == 2 and call(n=psk.PSK_MAX_VECTORS + 1) == 2 and call(ldy=47) == 2 and call(ldx=96) == 2 and call(ldy=2 ** 31) == 2
    assert call(ws=NULL) == 4 and call(ws=AT8) == 4 and call(have=255) == 4
    assert call(type=3) == 5 and call(type=-1) == 5
    for over in (dict(codes=264), dict(ld=120), dict(scales=258)):
        assert call(i8(**over)) == 7, over
    assert call(Y=ODD) == 7 and call(X=ODD) == 7 and call(bias=AT2) == 7


def test_products_refuse_more():
    assert psk.lib().psk_gemm_i8(None, 1, ONE, 112, ONE, NULL, 1, ONE, 48, ONE, BIG, NULL) == 1
    assert psk.lib().psk_linear_i8(None, 1, 1, ONE, 112, NULL, ONE, 48, ONE, BIG, NULL) == 1
    assert gemm(scales=NULL) == 1 and gemm(scales=AT2) == 7 and gemm(X=AT8) == 7 and gemm(ldx=120) == 7 and gemm(ldx=2 ** 23 + 16) == 2
    assert linear(have=psk.psk_linear_i8_workspace_bytes(48, 100, 4, psk.PSK_BF16) - 1) == 4
    assert gemm(have=psk.psk_gemm_i8_workspace_bytes(48, 100, 4) - 1) == 4
    assert psk.psk_gemm_i8_workspace_bytes(48, psk.PSK_I8_MAX_COLS + 1, 4) == 0 and psk.psk_gemm_i8_workspace_bytes(-1, 100, 4) == 0
    assert psk.psk_gemm_i8_workspace_bytes(48, 100, psk.PSK_MAX_VECTORS + 1) == 0
    assert psk.psk_linear_i8_workspace_bytes(48, 100, 4, 3) == 0 and psk.psk_linear_i8_workspace_bytes(48, -1, 4, 1) == 0


def embed(n=4, rows=48, dim=100, ids=ONE, type=psk.PSK_BF16, E=ONE, lde=100, ytype=psk.PSK_F32, Y=ONE, ldy=100):
    return psk.lib().psk_embed(n, rows, dim, ids, 1.0, type, E, lde, ytype, Y, ldy, NULL)


def embed_i8(E=None, n=4, ids=ONE, ytype=psk.PSK_F32, Y=ONE, ldy=100):
    E = i8() if E is None else E
    return psk.lib().psk_embed_i8(ctypes.byref(E), n, ids, 1.0, ytype, Y, ldy, NULL)


def test_embed_refuses():
    assert embed(n=0) == 0 and embed(dim=0, lde=0, ldy=0) == 0 and embed_i8(n=0) == 0
    assert psk.lib().psk_embed_i8(None, 1, ONE, 1.0, 0, ONE, 100, NULL) == 1
    for call in (embed, embed_i8):
        assert call(ids=NULL) == 1 and call(Y=NULL) == 1
        assert call(n=-1) == 2 and call(n=psk.PSK_MAX_TOKENS + 1) == 2 and call(ldy=99) == 2 and call(ldy=2 ** 31) == 2
        assert call(ytype=3) == 5 and call(ids=AT2) == 7 and call(Y=AT2) == 7 and call(ytype=psk.PSK_F16, Y=ODD) == 7
    assert embed(E=NULL) == 1 and embed(rows=-1) == 2 and embed(rows=2 ** 28) == 2 and embed(dim=-1) == 2 and embed(lde=99) == 2
    assert embed(dim=2 ** 28, lde=2 ** 28, ldy=2 ** 28) == 2 and embed(type=3) == 5 and embed(E=ODD) == 7
    assert embed_i8(i8(codes=0)) == 1 and embed_i8(i8(scales=0)) == 1 and embed_i8(i8(ld=96)) == 2 and embed_i8(i8(codes=264)) == 7 and embed_i8(i8(ld=120)) == 7


def grad(n=4, rows=48, dim=100, ids=ONE, type=psk.PSK_BF16, dY=ONE, ldy=100, gtype=psk.PSK_F32, dE=ONE, lde=100, accumulate=0, ws=ONE, have=BIG):
    return psk.lib().psk_embed_grad(n, rows, dim, ids, -1, 1.0, type, dY, ldy, gtype, dE, lde, accumulate, ws, have, NULL)


def test_embed_grad_refuses():
    assert grad(rows=0) == 0 and grad(dim=0, ldy=0, lde=0) == 0 and grad(n=0, accumulate=1) == 0
    for over in (dict(ids=NULL), dict(dY=NULL), dict(dE=NULL), dict(n=0, dE=NULL)):
        assert grad(**over) == 1, over
    for over in (dict(n=-1), dict(n=psk.PSK_MAX_TOKENS + 1), dict(rows=-1), dict(rows=2 ** 28), dict(dim=-1), dict(dim=2 ** 28, ldy=2 ** 28, lde=2 ** 28), dict(ldy=99),
                 dict(lde=99), dict(lde=2 ** 31)):
        assert grad(**over) == 2, over
    assert grad(ws=NULL) == 4 and grad(ws=AT8) == 4 and grad(have=psk.psk_embed_grad_workspace_bytes(4, 48, 100) - 1) == 4
    assert grad(type=3) == 5 and grad(gtype=psk.PSK_F16) == 5 and grad(type=psk.PSK_F32, gtype=psk.PSK_BF16) == 5
    for over in (dict(ids=AT2), dict(dY=ODD), dict(dE=AT2), dict(gtype=psk.PSK_BF16, dE=ODD)):
        assert grad(**over) == 7, over
    assert psk.psk_embed_grad_workspace_bytes(-1, 4, 4) == 0 and psk.psk_embed_grad_workspace_bytes(4, 4, 2 ** 28) == 0


def test_a_workspace_for_more_is_one_for_fewer():
    for rows, cols in ((1, 1), (300, 16384), (5003, 2051), (32768, 8192)):
        last = 0
        for n in (0, 1, 3, 4, 5, 17, 64, 300, 1000, 5000, 1 << 17, 1 << 19):
            b = psk.psk_gemm_i8_workspace_bytes(rows, cols, n)
            assert b >= max(last, 256)
            last = b
            assert psk.psk_linear_i8_workspace_bytes(rows, cols, n, psk.PSK_F16) >= b + n * cols
    for dim in (1, 3, 4, 64, 255, 257, 515, 1027, 4096, 9000):
        last = 0
        for n in list(range(0, 300)) + [2 ** k + d for k in range(9, 24) for d in (-1, 0, 1)] + [1 << 24]:
            b = psk.psk_embed_grad_workspace_bytes(n, 50000, dim)
            assert b >= last, (n, dim)
            last = b


def test_binding_refuses():
    codes, scales = torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8)
    for args in ((codes.int(), scales, 32), (codes, scales.half(), 32), (codes, scales[:7], 32), (codes, scales, 33), (codes[0], scales, 32),
                 (codes, torch.zeros(16)[::2], 32), (codes, scales, 32)):        # the last: on the host
        with pytest.raises(ValueError):
            psk.I8(*args)
    x, ids = torch.zeros(3, 20).half(), torch.zeros(3, dtype=torch.int32)
    for args in ((x, codes[:3, :16], scales[:3]), (x, codes[:2], scales[:3]), (x, codes[:3], scales[:2]), (x.double(), codes[:3], scales[:3]), (x[0], codes[:3], scales[:3]),
                 (x, codes[:3], scales[:3])):
        with pytest.raises(ValueError):
            psk.psk_quant_i8(*args)
    for args in ((ids.long(), x, x), (ids[:2], x, x), (ids, x, x[:, :8]), (ids, x.double(), x), (ids, x, x)):
        with pytest.raises(ValueError):
            psk.psk_embed(*args)
    for args in ((ids[:2], x, x), (ids, x[:2], x), (ids, x, x[:, :8]), (ids, x, x.double()), (ids, x, x)):
        with pytest.raises(ValueError):
            psk.psk_embed_grad(*args)
