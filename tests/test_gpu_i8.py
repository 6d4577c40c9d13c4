"""Products of 8-bit integers, and the tokens' quantisation, against the plain form in 64 bits."""
import numpy as np
import pytest

import ends_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def codes_of(rng, n, cols, pad=0, low=-127):
    """int8 rows in a multiple of 16 bytes, all bytes random (those behind the columns too)."""
    return torch.from_numpy(rng.integers(low, 128, (n, (cols + 15) // 16 * 16 + 16 * pad), dtype=np.int8))


def activations(rng, n, cols, dtype):
    x = rng.standard_normal((n, cols)) * np.where(rng.random((1, cols)) < 0.05, 10, 1)
    return torch.from_numpy(x).to(TYPES[dtype])


def guarded(n, rows, dtype, pad=5):
    buf = torch.full((n + 2, rows + pad), 77.0, dtype=TYPES[dtype], device="cuda")
    return buf, buf[1:n + 1, :rows]


def intact(buf, n, rows):
    torch.cuda.synchronize()
    return bool((buf[0] == 77).all()) and bool((buf[n + 1] == 77).all()) and bool((buf[:, rows:] == 77).all())


# ------------------------------------------------------------------ tokens in 8 bits
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,cols", [(1, 1), (3, 7), (2, 8), (5, 15), (4, 16), (7, 17), (33, 255), (3, 2048), (2, 2051), (5, 8191), (2, 8200), (1, 20000), (2, 131071)])
def test_quant(dtype, n, cols):
    rng = np.random.default_rng(n * 1000 + cols)
    x = activations(rng, n, cols, dtype)
    wide = torch.full((n, cols + 9), float("nan"), dtype=TYPES[dtype])
    wide[:, 3:3 + cols] = x
    room = (cols + 15) // 16 * 16
    codes, scales = torch.full((n, room + 16), 77, dtype=torch.int8, device="cuda"), torch.full((n + 1,), 77.0, device="cuda")
    psk.psk_quant_i8(wide.cuda()[:, 3:3 + cols], codes, scales[:n])
    q, s = R.quantised(x)
    got = codes.cpu().long()
    assert bool((got[:, :cols] == q).all()), "%d codes differ" % int((got[:, :cols] != q).sum())
    assert bool((got[:, cols:room] == 0).all()) and bool((got[:, room:] == 77).all()) and float(scales[n]) == 77
    assert torch.equal(scales[:n].cpu(), s)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_quant_at_the_borders(dtype):
    """Values in the middle between two codes, and next to it on both sides; the smallest and largest rows."""
    t = TYPES[dtype]
    half = torch.arange(-253, 254, dtype=torch.float64) / 2
    rows = [torch.cat([half, torch.tensor([127.0])])]                            # m = 127: every half is a tie
    for m in (1.0, 3.0, 0.7, 127.5, 1e-3):
        mid = torch.tensor(m, dtype=t).double() * half / 127
        near = mid.to(t)
        step = torch.finfo(t).eps * near.abs().double()
        rows += [torch.cat([v.double(), torch.tensor([m], dtype=t).double()]) for v in (near, (near.double() + step).to(t), (near.double() - step).to(t))]
    tiny, huge = torch.finfo(t).smallest_normal, torch.finfo(t).max
    for m in (tiny, tiny * torch.finfo(t).eps, tiny * torch.finfo(t).eps * 5, tiny * 200, huge, huge / 2):
        rows.append(torch.cat([half / 127 * m, torch.tensor([m], dtype=torch.float64)]))
    x = torch.stack(rows).to(t)
    codes, scales = torch.empty((x.shape[0], 512), dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], device="cuda")
    psk.psk_quant_i8(x.cuda(), codes, scales)
    q, s = R.quantised(x)
    assert bool((codes.cpu().long()[:, :x.shape[1]] == q).all()), "%d codes differ" % int((codes.cpu().long()[:, :x.shape[1]] != q).sum())
    assert torch.equal(scales.cpu(), s)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_is_not_finite_spoils_its_own_token(dtype):
    rng = np.random.default_rng(3)
    n, rows, cols = 7, 33, 70
    x = activations(rng, n, cols, dtype)
    x[1, 5], x[2, 69], x[4, 0], x[5] = float("inf"), float("nan"), float("-inf"), 0
    codes, scales = torch.empty((n, 80), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    psk.psk_quant_i8(x.cuda(), codes, scales)
    q, s = R.quantised(x)
    assert bool((codes.cpu().long()[:, :cols] == q).all()) and torch.equal(torch.isnan(scales.cpu()), torch.tensor([0, 1, 1, 0, 1, 0, 0]).bool())
    assert float(scales[5]) == 0
    w, a = codes_of(rng, rows, cols), torch.rand(rows)
    bias = torch.randn(rows)
    Y = torch.empty(n, rows, dtype=TYPES[dtype], device="cuda")
    for m in (n, 2):                                        # few and more tokens
        psk.psk_linear_i8(psk.I8(w.cuda(), a.cuda(), cols=cols), x[:m].cuda(), Y[:m], bias=bias.cuda())
        ref, bound = R.product(q[:m], w[:, :cols].long(), a, s[:m], bias, TYPES[dtype])
        R.check(Y[:m], ref, bound, "not finite " + dtype)


# ------------------------------------------------------------------ products
SIZES = [(1, 1, 1), (16, 16, 1), (17, 15, 2), (5, 17, 3), (40, 127, 4), (64, 128, 5), (33, 129, 16), (100, 255, 17), (50, 256, 31), (65, 257, 32), (130, 640, 33),
         (48, 1000, 64), (63, 1024, 65), (200, 300, 100), (257, 384, 127), (129, 130, 129), (300, 2051, 150), (255, 512, 255), (256, 513, 256), (300, 150, 257),
         (512, 200, 513), (270, 1100, 600), (515, 140, 1030), (1000, 64, 5), (3000, 48, 2), (7, 4100, 9), (20, 16400, 1), (19, 40000, 7), (3, 131071, 2), (5, 131071, 70)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,n", SIZES)
def test_products(dtype, rows, cols, n):
    rng = np.random.default_rng(rows * 7 + cols * 3 + n)
    w, a = codes_of(rng, rows, cols), torch.from_numpy(rng.uniform(0.5, 1, rows)).float() / cols
    A = psk.I8(w.cuda(), a.cuda(), cols=cols)
    bias = torch.randn(rows) if n % 2 else None
    b = None if bias is None else bias.cuda()
    q, s = codes_of(rng, n, cols, low=-128), torch.from_numpy(rng.uniform(0.5, 1, n)).float() / 50
    buf, Y = guarded(n, rows, dtype)
    psk.psk_gemm_i8(A, q.cuda(), s.cuda(), Y, bias=b)
    assert intact(buf, n, rows), "wrote past Y"
    ref, bound = R.product(q[:, :cols].long(), w[:, :cols].long(), a, s, bias, TYPES[dtype])
    R.check(Y, ref, bound, "gemm %s %dx%dx%d" % (dtype, rows, cols, n))

    x = activations(rng, n, cols, dtype)
    buf, Y = guarded(n, rows, dtype)
    psk.psk_linear_i8(A, x.cuda(), Y, bias=b)
    assert intact(buf, n, rows), "wrote past Y"
    ref, bound = R.product(*(lambda c: (c[0], w[:, :cols].long(), a, c[1], bias, TYPES[dtype]))(R.quantised(x)))
    R.check(Y, ref, bound, "linear %s %dx%dx%d" % (dtype, rows, cols, n))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 6, 40, 70, 300])
def test_strides_and_what_lies_behind_the_rows(dtype, n):
    """X at odd elements between NaN, rows of codes farther apart than they need and followed by other bytes, Y in a wider buffer at an odd place."""
    rng = np.random.default_rng(n)
    rows, cols = 75, 205
    w, a = codes_of(rng, rows, cols, pad=3), torch.rand(rows)
    q, s = codes_of(rng, n, cols, pad=1), torch.rand(n)
    wide = torch.full((n, cols + 11), float("nan"), dtype=TYPES[dtype])
    x = activations(rng, n, cols, dtype)
    wide[:, 3:3 + cols] = x
    A = psk.I8(w.cuda()[:, 16:], a.cuda(), cols=cols)       # begins 16 bytes into its buffer
    for what, (codes, scales) in (("gemm", (q[:, :cols].long(), s)), ("linear", R.quantised(x))):
        buf = torch.full((n, rows + 7), 77.0, dtype=TYPES[dtype], device="cuda")
        Y = buf[:, 3:3 + rows]
        if what == "gemm":
            psk.psk_gemm_i8(A, q.cuda(), s.cuda(), Y)
        else:
            psk.psk_linear_i8(A, wide.cuda()[:, 3:3 + cols], Y)
        ref, bound = R.product(codes, w[:, 16:16 + cols].long(), a, scales, None, TYPES[dtype])
        R.check(Y, ref, bound, "%s %s" % (what, dtype))
        assert bool((buf[:, :3] == 77).all()) and bool((buf[:, 3 + rows:] == 77).all())


@pytest.mark.parametrize("n", [1, 4, 5, 64, 65, 600])
def test_largest_sums(n):
    """Every product 2^14: sums that just fit 32 bits, and a difference of one in the last column."""
    cols, rows = 131071, 18
    w = torch.full((rows, 131072), -128, dtype=torch.int8)
    w[3, cols - 1], w[:, cols:] = 127, 55
    q = w[:1].repeat(n, 1)
    Y = torch.empty(n, rows, device="cuda")
    psk.psk_gemm_i8(psk.I8(w.cuda(), torch.ones(rows).cuda(), cols=cols), q.cuda(), torch.ones(n).cuda(), Y)
    ref = torch.full((n, rows), 2.0 ** 14 * cols, dtype=torch.float64)
    ref[:, 3] -= 128 * 255
    assert torch.equal(Y.cpu(), ref.float())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,n", [(301, 16384, 7), (13, 16385, 5), (70, 9000, 300), (1, 33000, 9), (600, 5000, 40), (255, 131071, 6), (18, 2200, 17), (30, 4500, 1500)])
def test_few_tiles_of_many_columns(dtype, rows, cols, n):
    """The columns in parts: several counts of steps to a part, parts that end in the middle of a step, rows that are no multiple of four."""
    test_products(dtype, rows, cols, n)


@pytest.mark.parametrize("rows,cols,n", [(9, 63488, 1), (9, 63489, 1), (30, 31744, 2), (30, 31745, 2), (21, 15872, 4), (21, 15873, 3), (5, 8, 4), (5, 7, 3), (2100, 1030, 1),
                                         (2040, 1024, 2), (2050, 700, 3), (9000, 24, 1), (1024, 7169, 1), (1025, 7169, 1), (1024, 7168, 2), (1021, 8200, 4), (3, 7169, 3)])
def test_where_the_way_for_few_tokens_changes(rows, cols, n):
    """The longest rows that it takes and the shortest, few and many rows, workgroups that take several tasks."""
    for dtype in ("bf16", "f32"):
        test_products(dtype, rows, cols, n)


@pytest.mark.parametrize("dtype,n", [("f16", 3500), ("f32", 1751)])
def test_results_larger_than_the_caches(dtype, n):
    """From 32 MB on these are stored past them; rows of Y that begin at odd places."""
    test_products(dtype, 5001, 40, n)


def test_a_workspace_for_more_tokens():
    """One that is made for many is enough for fewer, and what it held before does not matter."""
    rng = np.random.default_rng(12)
    rows, cols = 200, 9000
    w, a = codes_of(rng, rows, cols), torch.rand(rows) / cols
    A = psk.I8(w.cuda(), a.cuda(), cols=cols)
    x = activations(rng, 700, cols, "bf16")
    ws = psk.psk_linear_i8_workspace(A, x.cuda())
    for n in (700, 5, 90, 1, 300):
        ws.fill_(0xa5)
        Y = torch.empty(n, rows, dtype=torch.bfloat16, device="cuda")
        psk.psk_linear_i8(A, x[:n].cuda(), Y, ws=ws)
        q, s = R.quantised(x[:n])
        ref, bound = R.product(q, w[:, :cols].long(), a, s, None, torch.bfloat16)
        R.check(Y, ref, bound, "%d tokens" % n)


def test_no_columns_no_rows_no_tokens():
    bias, a = torch.randn(5).cuda(), torch.ones(5).cuda()
    A = psk.I8(torch.zeros((5, 0), dtype=torch.int8, device="cuda"), a, cols=0)
    for n in (1, 9, 300):
        Y = torch.full((n, 5), 77.0, device="cuda")
        psk.psk_linear_i8(A, torch.zeros((n, 0), device="cuda"), Y, bias=bias)
        assert bool((Y == bias).all())
        psk.psk_gemm_i8(A, torch.zeros((n, 0), dtype=torch.int8, device="cuda"), torch.ones(n).cuda(), Y)
        assert bool((Y == 0).all())
    A = psk.I8(torch.zeros((0, 16), dtype=torch.int8, device="cuda"), a[:0])
    assert psk.psk_linear_i8(A, torch.zeros((3, 16)).cuda(), torch.empty((3, 0), device="cuda")).numel() == 0
    A = psk.I8(torch.zeros((5, 16), dtype=torch.int8, device="cuda"), a)
    assert psk.psk_linear_i8(A, torch.zeros((0, 16)).cuda(), torch.empty((0, 5), device="cuda")).numel() == 0


def test_weights_quantised_by_rows():
    """psk_quant_i8 on a matrix of weights gives what I8 takes: within half a code of each weight, and the product of both."""
    rng = np.random.default_rng(8)
    w, x = torch.from_numpy(rng.standard_normal((70, 333))).float(), activations(rng, 9, 333, "f32")
    codes, scales = torch.empty((70, 336), dtype=torch.int8, device="cuda"), torch.empty(70, device="cuda")
    psk.psk_quant_i8(w.cuda(), codes, scales)
    back = codes.cpu()[:, :333].double() * scales.cpu().double()[:, None]
    # half a code, and the rounding of the scale times 127
    assert bool(((back - w.double()).abs() <= (0.5 + 127 * R.ULP) * scales.cpu().double()[:, None]).all())
    Y = torch.empty(9, 70, device="cuda")
    psk.psk_linear_i8(psk.I8(codes, scales, cols=333), x.cuda(), Y)
    q, s = R.quantised(x)
    ref, bound = R.product(q, codes.cpu()[:, :333].long(), scales.cpu(), s, None, torch.float32)
    R.check(Y, ref, bound, "weights by rows")


def test_offsets_past_32_bits():
    """Tokens, weights and results whose last rows lie more than 2^32 bytes or elements in."""
    far, cols, rows, n = 1 << 23, 64, 600, 300
    room = torch.zeros(rows * far, dtype=torch.int8, device="cuda")              # 5 GB
    w = room.as_strided((rows, cols), (far, 1))
    rng = np.random.default_rng(4)
    codes = codes_of(rng, rows, cols)
    w.copy_(codes)
    a, s, q = torch.rand(rows), torch.rand(n), codes_of(rng, n, cols)
    out = torch.empty(n * (1 << 24), dtype=torch.float16, device="cuda")         # 10 GB
    Y = out.as_strided((n, rows), (1 << 24, 1))
    psk.psk_gemm_i8(psk.I8(w, a.cuda()), q.cuda(), s.cuda(), Y)
    ref, bound = R.product(q.long(), codes.long(), a, s, None, torch.float16)
    R.check(Y, ref, bound, "far")
    psk.psk_gemm_i8(psk.I8(q.cuda(), s.cuda()), w, a.cuda(), Y.as_strided((rows, n), (1 << 22, 1)))
    ref, bound = R.product(codes.long(), q.long(), s, a, None, torch.float16)
    R.check(Y.as_strided((rows, n), (1 << 22, 1)), ref, bound, "far tokens")
