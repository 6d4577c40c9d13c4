"""Products with 4-bit weights against the plain form in 64 bits."""
import ctypes

import numpy as np
import pytest

import serving_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def dev(*ts):
    return [None if t is None else t.cuda() for t in ts]


def product(w, x, cols, group, ldy=None):
    """psk_gemm_q4 into a buffer with guards around Y's rows; returns Y."""
    n, rows = x.shape[0], w[0].shape[0]
    A = psk.Q4(*dev(*w), cols=cols, group=group)
    pad = 0 if ldy is None else ldy - rows
    buf = torch.full((n + 2, rows + pad), 77.0, dtype=x.dtype, device="cuda")
    Y = buf[1:n + 1, :rows]
    psk.psk_gemm_q4(A, x, Y)
    torch.cuda.synchronize()
    assert bool((buf[0] == 77).all()) and bool((buf[n + 1] == 77).all()) and bool((buf[:, rows:] == 77).all()), "wrote past Y"
    return Y


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,n,group,zeros,scale32", [
    (1, 1, 1, 32, False, False), (16, 32, 1, 32, True, False), (17, 31, 2, 32, True, True), (15, 33, 5, 64, False, False),
    (40, 127, 6, 128, True, False), (33, 128, 16, 64, False, True), (100, 129, 17, 32, True, False), (64, 1000, 3, 128, True, True),
    (50, 2051, 1, 64, True, False), (48, 4100, 33, 256, False, False), (20, 640, 64, 32, True, False), (35, 300, 65, 4096, True, False),
    (18, 1100, 130, 128, False, False), (8, 16400, 1, 128, True, False)])
def test_products(dtype, rows, cols, n, group, zeros, scale32):
    t = TYPES[dtype]
    rng = np.random.default_rng(rows * 1000 + cols)
    w = R.q4_weights(rng, rows, cols, group, zeros, torch.float32 if scale32 else t)
    x = torch.from_numpy(rng.standard_normal((n, cols))).to(t)
    ref, bound = R.gemm(R.dequantised(*w, cols, group), x, t)
    R.check(product(w, x.cuda(), cols, group), ref, bound, "%s %dx%dx%d" % (dtype, rows, cols, n))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,n,group,zeros,scale32", [
    (37, 255, 5, 32, True, False), (65, 1024, 16, 64, False, False), (16, 1025, 17, 32, True, True), (130, 2047, 5, 128, True, False),
    (33, 2048, 33, 512, True, False), (17, 2049, 48, 32, False, False), (5000, 1056, 6, 256, True, False), (47, 4096, 16, 4096, True, True),
    (31, 4095, 21, 64, True, False), (40, 4097, 5, 32, True, False), (40, 4097, 40, 128, False, True), (9000, 100, 17, 128, True, False)])
def test_where_the_way_for_more_vectors_changes(dtype, rows, cols, n, group, zeros, scale32):
    """Columns on both sides of every length at which another kernel or another number of waves takes over, few and many sets of rows."""
    test_products(dtype, rows, cols, n, group, zeros, scale32)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("cols", [512, 2048, 2600, 4099])
@pytest.mark.parametrize("group", [32, 64, 128, 256, 512, 1024, 1 << 30])
def test_every_group_with_few_and_more_vectors(dtype, cols, group):
    """Groups smaller and larger than what a wave takes at once, short and long rows."""
    for n, zeros in ((1, True), (4, False), (7, True)):
        test_products(dtype, 19, cols, n, group, zeros, False)


def test_very_many_vectors():
    rng = np.random.default_rng(10)
    w = R.q4_weights(rng, 17, 40, 32, True, torch.float16)
    x = torch.from_numpy(rng.standard_normal((200001, 40))).half()
    ref, bound = R.gemm(R.dequantised(*w, 40, 32), x, torch.float16)
    R.check(product(w, x.cuda(), 40, 32), ref, bound, "200001 vectors")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_strides_and_what_lies_behind_the_rows(dtype):
    """Rows of X that start at odd elements between NaN, rows of codes and scales farther apart than they need, Y in a wider buffer."""
    t, rows, cols, n, group = TYPES[dtype], 37, 205, 7, 64
    rng = np.random.default_rng(5)
    codes, scales, zeros = R.q4_weights(rng, rows, cols, group, True, t, pad=2)
    wide = torch.full((rows, 9), float("nan"), dtype=t)
    wz = torch.full((rows, 9), 200, dtype=torch.uint8)
    wide[:, 2:6], wz[:, 2:6] = scales, zeros
    buf = torch.full((n, cols + 11), float("nan"), dtype=t)
    x = torch.from_numpy(rng.standard_normal((n, cols))).to(t)
    buf[:, 3:3 + cols] = x
    ref, bound = R.gemm(R.dequantised(codes, scales, zeros, cols, group), x, t)
    ws, wzd, xd = wide.cuda(), wz.cuda(), buf.cuda()
    y = torch.full((n, rows + 5), 77.0, dtype=t, device="cuda")
    A = psk.Q4(codes.cuda(), ws[:, 2:6], wzd[:, 2:6], cols=cols, group=group)
    psk.psk_gemm_q4(A, xd[:, 3:3 + cols], y[:, :rows])
    R.check(y[:, :rows], ref, bound, "strided " + dtype)
    assert bool((y[:, rows:] == 77).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_special_values(dtype):
    """An infinity or NaN spoils its own vector only, and only where the plain form is spoiled; zero points up to 255; a scale that is
    infinite spoils its own row."""
    t, rows, cols, n, group = TYPES[dtype], 33, 165, 9, 32
    rng = np.random.default_rng(6)
    codes, scales, zeros = R.q4_weights(rng, rows, cols, group, True, t)
    zeros[3] = 255
    scales[5, -1] = float("inf")
    x = torch.from_numpy(rng.standard_normal((n, cols))).to(t)
    x[1, 17], x[2, 40], x[4, 164] = float("inf"), float("nan"), float("-inf")
    x[6] = 0
    x[7, 3], x[7, 4] = torch.finfo(t).max, -torch.finfo(t).max
    x[8] = torch.finfo(t).smallest_normal * 8
    w = R.dequantised(codes, scales, zeros, cols, group)
    ref, bound = R.gemm(w, x, t)
    ref = ref.to(t).double() if dtype != "f32" else ref
    over = ref.abs() > torch.finfo(t).max
    ref[over] = torch.sign(ref[over]) * float("inf")
    got = product((codes, scales, zeros), x.cuda(), cols, group)
    # the row with the infinite scale is NaN or infinite as the signs of its last group fall: compared by itself
    keep = [i for i in range(rows) if i != 5]
    R.check(got[:, keep], ref[:, keep], bound[:, keep], "special " + dtype)
    assert not bool(torch.isfinite(got[:6, 5]).any())


@pytest.mark.parametrize("dtype,scale32", [("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("n,cols,group", [(1, 300, 32), (3, 2200, 256), (6, 300, 64), (20, 1500, 128), (5, 2600, 32), (20, 5000, 64)])
def test_scales_near_the_largest_number(dtype, scale32, n, cols, group):
    """Scales of 2^118 to 2^127 with activations of about 2^-100; a group of every row has weights that are all zero."""
    t, rows = TYPES[dtype], 35
    rng = np.random.default_rng(cols)
    codes, scales, _ = R.q4_weights(rng, rows, cols, group, False, torch.float32 if scale32 else t)
    scales[:] = 2.0 ** torch.from_numpy(rng.integers(118, 126, scales.shape)).double()
    scales[:, 1] = torch.finfo(scales.dtype).max
    codes[:, group // 2:group] = 0x88
    x = (torch.from_numpy(rng.standard_normal((n, cols))) * 2.0 ** -100).to(t)
    ref, bound = R.gemm(R.dequantised(codes, scales, None, cols, group), x, t)
    R.check(product((codes, scales, None), x.cuda(), cols, group), ref, bound, "large scales")


@pytest.mark.parametrize("n", [1, 6, 20])
@pytest.mark.parametrize("cols", [300, 5000])
def test_activations_below_the_smallest_normal_f16(n, cols):
    rng = np.random.default_rng(11)
    w = R.q4_weights(rng, 20, cols, 64, True, torch.float16, scale=50)
    x = torch.from_numpy(rng.standard_normal((n, cols)) * 5e-6).half()
    ref, bound = R.gemm(R.dequantised(*w, cols, 64), x, torch.float16)
    R.check(product(w, x.cuda(), cols, 64), ref, bound, "denormal activations")


def test_vectors_of_32_bits_keep_their_bits():
    """Values whose low bits matter: sums that cancel to the last bits of the activations."""
    rows, cols = 16, 256
    codes = torch.zeros(rows, 128, dtype=torch.uint8)
    codes[:, :] = 0x79                                     # even columns +1, odd ones -1
    scales = torch.ones(rows, 2)
    a = torch.from_numpy(np.random.default_rng(7).uniform(1, 2, 128)).float()
    x = torch.empty(1, cols)
    x[0, 0::2], x[0, 1::2] = torch.nextafter(a, a + 1), a
    ref = (x[0, 0::2].double() - x[0, 1::2].double()).sum()
    got = product((codes, scales, None), x.cuda(), cols, 128)[0, 0].item()
    # parts of 8 bits: the first ones and the second ones cancel exactly pair by pair or leave steps of 2^-23, all sums are below
    # 2^9 and multiples of 2^-23 where they are not exact: 2^-23 2^9 2^-23 per term at the very most
    assert abs(got - float(ref)) <= 256 * 2.0 ** -14 * 2.0 ** -23 * 2 ** 9, (got, float(ref))


@pytest.mark.parametrize("power", [0, -109])
@pytest.mark.parametrize("rows,cols,n", [(20, 300, 1), (20, 2500, 4), (20, 512, 5), (20, 1000, 33), (20, 1536, 16), (20, 2040, 5), (20, 2560, 16), (20, 5000, 33),
                                         (1500, 2560, 33)])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
def test_every_way_keeps_the_bits_of_vectors_of_32_bits(rows, cols, n, group, power):
    """Neighbouring numbers cancel to their last bits: rows of +1 -1 or -1 +1 by pairs of columns, each worth a step of 2^-23."""
    rng = np.random.default_rng(cols + n)
    signs = rng.integers(0, 2, (rows, cols // 2))
    codes = torch.zeros(rows, (cols + 31) // 32 * 16, dtype=torch.uint8)
    codes[:, :cols // 2] = torch.from_numpy(np.where(signs, 0x79, 0x97).astype(np.uint8))      # +1 -1, -1 +1
    scales = torch.full((rows, (cols + group - 1) // group), 2.0 ** min(100, -power))
    a = torch.from_numpy(rng.uniform(1, 2, (n, cols // 2)) * (1 - 2 * rng.integers(0, 2, (n, cols // 2)))).float()
    x = torch.empty(n, cols)
    x[:, 0::2], x[:, 1::2] = torch.nextafter(a, 2 * a), a
    d = (x[:, 0::2] - x[:, 1::2]).double()
    ref = d @ torch.from_numpy(2.0 * signs - 1).t()
    got = product((codes, scales, None), (x * 2.0 ** power).cuda(), cols, group).cpu().double() * 2.0 ** -(power + min(100, -power))
    # the sums of each part are multiples of its last bit, 2^-7, 2^-15 and 2^-23, and of 32 products below 2^6, 2^-2 and 2^-10; those of all three, of a
    # group and of the row, multiples of 2^-23 below 2: everything is exact
    assert torch.equal(got, ref), float((got - ref).abs().max() / ref.abs().max())


def test_empty_products():
    x = torch.zeros(3, 64, device="cuda", dtype=torch.float16)
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8, device="cuda"), torch.ones(8, 2, device="cuda", dtype=torch.float16)
    A = psk.Q4(codes, scales, cols=64, group=32)
    psk.psk_gemm_q4(A, x[:0], torch.empty(0, 8, device="cuda", dtype=torch.float16))
    psk.psk_gemm_q4(psk.Q4(codes[:0], scales[:0], cols=64, group=32), x, torch.empty(3, 0, device="cuda", dtype=torch.float16))
    y = torch.full((3, 8), 5.0, device="cuda", dtype=torch.float16)
    psk.psk_gemm_q4(psk.Q4(codes, scales[:, :0], cols=0, group=32), x[:, :0], y)
    assert bool((y == 0).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n", [1, 4, 5, 17, 70000])
def test_products_without_columns(dtype, n):
    """No columns: rows of zeros for any number of vectors, nothing behind them, and no codes, scales or vectors needed for it."""
    t, rows = TYPES[dtype], 37
    d = psk.psk_q4()
    d.count, d.rows, d.cols, d.group, d.scale_type = 1, rows, 0, 64, psk.PSK_F32
    types = {"f32": psk.PSK_F32, "f16": psk.PSK_F16, "bf16": psk.PSK_BF16}
    y = torch.full((n + 1, rows + 3), 5.0, device="cuda", dtype=t)
    ws = torch.empty(psk.psk_gemm_q4_workspace_bytes(rows, 0, n, types[dtype]), device="cuda", dtype=torch.uint8)
    st = psk.lib().psk_gemm_q4(ctypes.byref(d), n, types[dtype], None, 0, y.data_ptr(), rows + 3, ws.data_ptr(), ws.numel(),
                               torch.cuda.current_stream().cuda_stream)
    assert st == 0
    assert bool((y[:n, :rows] == 0).all()) and bool((y[:, rows:] == 5).all()) and bool((y[n] == 5).all())
    codes, scales = torch.zeros(rows, 0, dtype=torch.uint8, device="cuda"), torch.zeros(rows, 0, device="cuda", dtype=t)
    whole = torch.full((n, rows), 5.0, device="cuda", dtype=t)
    psk.psk_gemm_q4(psk.Q4(codes, scales, cols=0, group=64), torch.zeros(n, 0, device="cuda", dtype=t), whole)
    assert bool((whole == 0).all())


@pytest.mark.parametrize("rows,cols,n", [((1 << 20) + 37, 8192 + 64, 3), ((1 << 20) + 37, 8192 + 64, 20), ((1 << 21) + (1 << 17) + 37, 4096, 5)])
def test_codes_beyond_four_gigabytes(rows, cols, n):
    """A vocabulary's worth of rows whose offsets pass 32 bits; the first and last rows and some in between are checked."""
    group = 128
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    codes = torch.randint(0, 256, (rows, (cols + 31) // 32 * 16), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.rand(rows, (cols + group - 1) // group, generator=g, device="cuda").to(torch.bfloat16)
    x = torch.randn(n, cols, generator=g, device="cuda").to(torch.bfloat16)
    y = torch.zeros(n, rows, device="cuda", dtype=torch.bfloat16)
    psk.psk_gemm_q4(psk.Q4(codes, scales, cols=cols, group=group), x, y)
    torch.cuda.synchronize()
    for r in (0, 12345, (1 << 31) // codes.shape[1], (1 << 32) // codes.shape[1] + 1, rows - 16):
        part = slice(r, r + 16)
        ref, bound = R.gemm(R.dequantised(codes[part].cpu(), scales[part].cpu(), None, cols, group), x.cpu(), torch.bfloat16)
        R.check(y[:, part], ref, bound, "rows from %d" % r)


@pytest.mark.parametrize("n", [1, 5])
def test_as_many_rows_as_a_matrix_may_have(n):
    rows, cols, group = (1 << 28) - 256, 32, 32
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    codes = torch.randint(0, 256, (rows, 16), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.rand(rows, 1, generator=g, device="cuda", dtype=torch.float16)
    x = torch.randn(n, cols, generator=g, device="cuda").half()
    y = torch.zeros(n, rows, device="cuda", dtype=torch.float16)
    psk.psk_gemm_q4(psk.Q4(codes, scales, cols=cols, group=group), x, y)
    torch.cuda.synchronize()
    for r in (0, rows // 2 + 3, rows - 17):
        part = slice(r, r + 17)
        ref, bound = R.gemm(R.dequantised(codes[part].cpu(), scales[part].cpu(), None, cols, group), x.cpu(), torch.float16)
        R.check(y[:, part], ref, bound, "rows from %d" % r)


@pytest.mark.parametrize("n", [1, 20])
def test_other_stream_and_graph(n):
    """On a stream that is not the current one, and captured: replays follow the activations, with eager work in between."""
    rng = np.random.default_rng(8)
    rows, cols, group = 200, 600, 128
    w = R.q4_weights(rng, rows, cols, group, True, torch.float16)
    A = psk.Q4(*dev(*w), cols=cols, group=group)
    x = torch.zeros(n, cols, dtype=torch.float16, device="cuda")
    y = torch.zeros(n, rows, dtype=torch.float16, device="cuda")
    ws = psk.psk_gemm_q4_workspace(A, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    psk.psk_gemm_q4(A, x, y, ws=ws, stream=side)
    psk.psk_gemm_q4(A, x, y, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        psk.psk_gemm_q4(A, x, y, ws=ws)
    for rep in range(4):
        xh = torch.from_numpy(rng.standard_normal((n, cols))).half()
        x.copy_(xh)
        y.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        ref, bound = R.gemm(R.dequantised(*w, cols, group), xh, torch.float16)
        R.check(y, ref, bound, "replay %d" % rep)
        eager = torch.zeros_like(y)
        psk.psk_gemm_q4(A, x, eager)
        assert torch.equal(eager, y)


def test_results_do_not_change_from_run_to_run():
    rng = np.random.default_rng(9)
    w = R.q4_weights(rng, 500, 3000, 64, True, torch.bfloat16)
    x = torch.from_numpy(rng.standard_normal((11, 3000))).bfloat16().cuda()
    first = product(w, x, 3000, 64).clone()
    for _ in range(5):
        assert torch.equal(first, product(w, x, 3000, 64))
    # a vector's result does not depend on the ones beside it, as long as the same kernel takes it
    assert torch.equal(first[4:9], product(w, x[4:9], 3000, 64))
