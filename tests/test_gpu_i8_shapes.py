"""Products of 8-bit integers in each shape of tile, over all columns and over parts of them.  (tests/test_i8_plan.py looks after the sizes.)"""
import numpy as np
import pytest

import ends_ref as R
from test_gpu_i8 import TYPES, codes_of, guarded, intact

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402

# rows, cols, n: more steps of 128 columns than the shape has stages, a last one that ends within 16 bytes, partial tiles of tokens and of channels
WHOLE = [(17, 1159, 17), (2119, 1157, 17), (33, 1045, 2065), (4097, 659, 33), (132, 653, 2746), (4117, 659, 98), (4313, 653, 202), (4111, 655, 392), (4176, 525, 901),
         (2567, 399, 3091)]
PARTS = [(18, 4102, 17), (257, 8194, 17), (33, 6595, 259), (514, 4489, 33), (18, 4581, 1031), (34, 4564, 1037), (32, 4871, 2069), (66, 10085, 1029), (66, 17237, 4156)]


def compare(dtype, rows, cols, n):
    rng = np.random.default_rng(rows * 7 + cols * 3 + n)
    w, a = codes_of(rng, rows, cols), torch.from_numpy(rng.uniform(0.5, 1, rows)).float() / cols
    q, s = codes_of(rng, n, cols, low=-128), torch.from_numpy(rng.uniform(0.5, 1, n)).float() / 50
    bias = torch.from_numpy(rng.standard_normal(rows)).float()
    buf, Y = guarded(n, rows, dtype)
    psk.psk_gemm_i8(psk.I8(w.cuda(), a.cuda(), cols=cols), q.cuda(), s.cuda(), Y, bias=bias.cuda())
    assert intact(buf, n, rows), "wrote past Y"
    ref, bound = R.product(q[:, :cols].long(), w[:, :cols].long(), a, s, bias, TYPES[dtype])
    R.check(Y, ref, bound, "gemm %s %dx%dx%d" % (dtype, rows, cols, n))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,n", WHOLE)
def test_shapes_over_all_columns(dtype, rows, cols, n):
    compare(dtype, rows, cols, n)


@pytest.mark.parametrize("rows,cols,n", PARTS)
def test_shapes_over_parts_of_the_columns(rows, cols, n):
    """Sums are whole numbers whatever the type of Y."""
    compare("f32", rows, cols, n)
