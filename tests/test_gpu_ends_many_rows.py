"""More rows than a grid has workgroups: tables that are quantised, tokens that are looked up."""
import numpy as np
import pytest

import ends_ref as R
from test_gpu_i8 import TYPES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402


def normal(n, cols, dtype):
    x = torch.randn(n, cols, generator=torch.Generator(device="cuda").manual_seed(n + cols), device="cuda").to(TYPES[dtype])
    x[1::1000] = 0
    x[2::1000, 0] = float("nan")
    return x


def quantised(x):
    n, cols = x.shape
    codes, scales = torch.full((n, (cols + 15) // 16 * 16), 77, dtype=torch.int8, device="cuda"), torch.full((n,), 77.0, device="cuda")
    psk.psk_quant_i8(x, codes, scales)
    return codes, scales


def same(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("n,cols,dtype", [(131075, 20, "f16"), (131072, 64, "bf16"), (65537, 300, "f32"), (16_777_219, 3, "bf16")])
def test_tables(n, cols, dtype):
    """A workgroup takes one row and then another, a thread one short row and then another; every 50th row and the last against the plain form."""
    x = normal(n, cols, dtype)
    codes, scales = quantised(x)
    at = torch.cat([torch.arange(0, n, 50 if n < 1 << 20 else 5000), torch.arange(n - 10, n)])
    q, s = R.quantised(x[at.cuda()].cpu())
    assert bool((codes[at.cuda(), :cols].cpu().long() == q).all()) and bool((codes[:, cols:] == 0).all()) and same(scales[at.cuda()].cpu(), s)
    # all rows against calls of fewer of them
    for first in range(0, n, 50000 if n < 1 << 20 else 9_000_000):
        part = slice(first, min(n, first + (50000 if n < 1 << 20 else 9_000_000)))
        c, s = quantised(x[part])
        assert torch.equal(codes[part], c) and same(scales[part], s)


@pytest.mark.parametrize("cols", [2100, 4100, 8300])
def test_long_rows(cols):
    """Rows whose pieces stay in registers between the two passes, and rows longer than that."""
    x = normal(65541, cols, "bf16")
    codes, scales = quantised(x)
    for first in (0, 30000, 60000):
        c, s = quantised(x[first:first + 30000])
        assert torch.equal(codes[first:first + 30000], c) and same(scales[first:first + 30000], s)


@pytest.mark.parametrize("table,dtype,dim", [("f16", "f16", 1030), ("bf16", "f32", 1025), ("i8", "bf16", 2049)])
def test_tokens(table, dtype, dim):
    n, rows = 65541, 3001
    ids = torch.from_numpy(np.random.default_rng(dim).integers(-5, rows + 5, n).astype(np.int32)).cuda()
    known = (ids >= 0) & (ids < rows)
    at = ids.clamp(0, rows - 1).long()
    g = torch.Generator(device="cuda").manual_seed(dim)
    if table == "i8":
        codes = torch.randint(-128, 128, (rows, (dim + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)
        scales = torch.rand(rows, generator=g, device="cuda")
        E, want = psk.I8(codes, scales, cols=dim), codes[:, :dim].float() * scales[:, None]
    else:
        E = torch.randn(rows, dim, generator=g, device="cuda").to(TYPES[table])
        want = E.float()
    buf = torch.full((n + 1, dim + 1), 77.0, dtype=TYPES[dtype], device="cuda")
    psk.psk_embed(ids, E, buf[:n, :dim])
    # a product with 1, or of a code and its scale, is rounded once to 32 bits at most, and a 16-bit result from there
    want = want.to(TYPES[dtype])
    for first in range(0, n, 8192):
        part = slice(first, min(n, first + 8192))
        assert torch.equal(buf[part, :dim], torch.where(known[part, None], want[at[part]], torch.zeros((), dtype=TYPES[dtype], device="cuda")))
    assert bool((buf[n] == 77).all()) and bool((buf[:, dim] == 77).all())
