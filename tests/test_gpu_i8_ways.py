"""Every way of a product of 8-bit integers gives the same bits: few tokens, tiles, columns in parts, codes given or made in the call."""
import numpy as np
import pytest

from test_gpu_i8 import TYPES, activations, codes_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402


def rounded(A, q, s, bias, dtype):
    """The sum in 32 bits, its product with the channel's scale in 32 bits, and the fused multiply-add, to f16 and f32 at once (the product of two numbers of 32
    bits is exact in 64, and so is the sum without bias)."""
    sums = (q[:, :A.cols].double() @ A.codes[:, :A.cols].double().t()).cpu().numpy().astype(np.float32)
    y = (sums * A.scales.cpu().numpy()).astype(np.float64) * s.cpu().numpy().astype(np.float64)[:, None]
    if bias is not None:
        y = y + bias.cpu().numpy().astype(np.float64)
    y = torch.from_numpy(y.astype(np.float16 if dtype == "f16" else np.float32))
    return y.to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("rows,cols", [(301, 9000), (515, 300), (1100, 7200), (9, 20)])
def test_the_same_bits(dtype, with_bias, rows, cols):
    """Tokens of a batch one to four at a time, five (columns in parts where they are many), and all; and the roundings that the results are made by."""
    rng = np.random.default_rng(rows + cols)
    n = 600 if rows < 1000 else 300
    w, q = codes_of(rng, rows, cols).cuda(), codes_of(rng, n, cols, low=-128).cuda()
    a, s = (torch.from_numpy(rng.uniform(0.5, 1, k)).float().cuda() / 100 for k in (rows, n))
    bias = torch.from_numpy(rng.standard_normal(rows) * cols ** 0.5 / 2).float().cuda() if with_bias else None
    A = psk.I8(w, a, cols=cols)

    def product(first, count, t=dtype):
        return psk.psk_gemm_i8(A, q[first:first + count], s[first:first + count], torch.empty(count, rows, dtype=TYPES[t], device="cuda"), bias=bias)
    whole = product(0, n)
    for count, begins in ((1, (0, 7, n - 1)), (2, (3,)), (3, (11,)), (4, (0, n - 4)), (5, (0, 20)), (17, (1,)), (70, (30,)), (200, (64,))):
        for first in begins:
            assert torch.equal(product(first, count), whole[first:first + count]), (first, count)
    assert torch.equal(rounded(A, q, s, bias, dtype), whole.cpu())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(301, 9000), (515, 300), (70, 5)])
def test_the_same_bits_from_activations(dtype, rows, cols):
    rng = np.random.default_rng(rows * 3 + cols)
    n = 300
    A = psk.I8(codes_of(rng, rows, cols).cuda(), torch.from_numpy(rng.uniform(0.5, 1, rows)).float().cuda() / 100, cols=cols)
    x = activations(rng, n, cols, dtype).cuda()
    codes, scales = torch.empty((n, (cols + 15) // 16 * 16), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    psk.psk_quant_i8(x, codes, scales)
    whole = psk.psk_gemm_i8(A, codes, scales, torch.empty(n, rows, dtype=TYPES[dtype], device="cuda"))
    for first, count in ((0, 1), (299, 1), (5, 2), (6, 3), (8, 4), (0, 5), (40, 60), (0, n)):
        got = psk.psk_linear_i8(A, x[first:first + count], torch.empty(count, rows, dtype=TYPES[dtype], device="cuda"))
        assert torch.equal(got, whole[first:first + count]), (first, count)
