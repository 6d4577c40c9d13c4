"""The gradient of the embedding lookup in each of its ways: one launch, ranges of rows, digits counted by each workgroup, digits scanned."""
import numpy as np
import pytest

import ends_ref as R
from test_gpu_embed import TYPES, gradient, ints, tokens

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def expected(ids, dy, rows, factor, padding, dtype, old=None):
    """(dE, bound) as ends_ref.embed_grad, for many tokens at a time."""
    keep = (ids >= 0) & (ids < rows) & (ids != padding)
    at, v = ids[keep].long(), dy[keep].double()
    de, size = (torch.zeros(rows, dy.shape[1], dtype=torch.float64).index_add_(0, at, t) for t in (v, v.abs()))
    count = torch.bincount(at, minlength=rows)[:, None].double()
    y = de * factor if old is None else old.double() + de * factor
    # the plain form adds up in 64 bits, in any order: count 2^-53 of the sizes
    bound = (count + 2) * R.ULP * size * abs(factor) + 2 * R.ULP * y.abs() + R.out_error(y, dtype) + count * 2.0 ** -53 * size * abs(factor)
    return y, bound if old is None else torch.where(count > 0, bound, torch.full_like(bound, 1e-300))


@pytest.mark.parametrize("n", [900, 3000, 70001])
def test_tokens_at_the_ends_of_their_type(n):
    """-2^31 and its neighbours, 2^31 - 1, the number of rows and the one before it, among rows of every range."""
    rng = np.random.default_rng(n)
    rows, dim = 5000, 8
    ends = np.array([-2 ** 31, -2 ** 31 + 1, -2 ** 31 + rows, -1, 0, 1, rows - 1, rows, rows + 1, 2 ** 31 - 1 - rows, 2 ** 31 - 1])
    ids = ints(np.where(rng.random(n) < 0.5, ends[rng.integers(0, len(ends), n)], rng.integers(0, rows, n)).astype(np.int32))
    dy = torch.from_numpy(rng.standard_normal((n, dim))).float()
    for padding in (-1, -2 ** 31, 2 ** 31 - 1, rows - 1):
        R.check(gradient(ids, dy, rows, "f32", padding=padding), *expected(ids, dy, rows, 1.0, padding, torch.float32), "ends, padding %d" % padding)


# n, rows, dim.  (tests/test_embed_plan.py looks after the sizes.)
RANGES = [(1100, 300, 250), (1500, 40, 512), (1100, 300, 300), (2100, 700, 1000), (1300, 90, 4099), (3000, 500, 600), (2049, 60, 2301)]
DIGITS = [(65537, 300, 8), (140001, 5000, 20), (262144, 300, 3), (262144, 200001, 5), (1030, 524289, 300)]
SCANNED = [(262145, 300, 8), (262145, 200001, 4), (300000, 600001, 3), (262200, 700, 300)]
PAIRS = [("f32", "f32"), ("f16", "f16"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32")]


def compare(dtype, gtype, n, rows, dim, kind, padding):
    rng = np.random.default_rng(n + 3 * rows + dim)
    ids = tokens(rng, n, rows, kind)
    dy = torch.randn(n, dim, generator=torch.Generator().manual_seed(n + dim)).to(TYPES[dtype])
    R.check(gradient(ids, dy, rows, gtype, 1.5, padding), *expected(ids, dy, rows, 1.5, padding, TYPES[gtype]), "assigned")
    old = torch.randn(rows, dim, generator=torch.Generator().manual_seed(rows)).to(TYPES[gtype])
    R.check(gradient(ids, dy, rows, gtype, 1.5, padding, old), *expected(ids, dy, rows, 1.5, padding, TYPES[gtype], old), "added")


@pytest.mark.parametrize("dtype,gtype", PAIRS)
@pytest.mark.parametrize("kind", ["head", "zipf"])
@pytest.mark.parametrize("n,rows,dim", RANGES)
def test_ranges_of_rows(dtype, gtype, kind, n, rows, dim):
    """One to three pieces of 256 columns to a wave, one and several such waves to a row, rows over many tiles."""
    compare(dtype, gtype, n, rows, dim, kind, rows // 3)


@pytest.mark.parametrize("dtype,gtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("n,rows,dim", DIGITS + SCANNED)
def test_digits(dtype, gtype, n, rows, dim):
    """On both sides of the border to counts that are scanned; keys of one to three digits."""
    compare(dtype, gtype, n, rows, dim, "head" if n % 2 else "zipf", -1)


def test_as_many_tokens_as_there_may_be():
    """2^24 tokens, a quarter of them one; sums of small whole numbers, which are exact."""
    n, rows, dim = 1 << 24, 1000003, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(-1000, rows + 1000, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand(n, generator=g, device="cuda") < 0.25] = 77777
    dy = torch.randint(-1, 2, (n, dim), generator=g, device="cuda").to(torch.bfloat16)
    got = gradient(ids.cpu(), dy.cpu(), rows, "f32")
    keep = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, dim, dtype=torch.int64).index_add_(0, ids[keep].cpu().long(), dy[keep].cpu().long())
    assert int(want.abs().max()) < 1 << 24 and torch.equal(got.cpu().long(), want)


def test_more_rows_to_clear_than_a_grid_has_workgroups():
    n, rows, dim = 70001, 17_000_001, 3
    ids = ints(np.random.default_rng(4).integers(0, rows, n))
    got = gradient(ids, torch.ones(n, dim), rows, "f32", pad=1)
    assert torch.equal(got[:, 1].cpu().long(), torch.bincount(ids.long(), minlength=rows))


@pytest.mark.parametrize("n,rows,dim", [(700, 300, 20), (3000, 300, 20), (70001, 300, 8), (262145, 5000, 4)])
def test_each_way_captured_and_replayed_with_new_tokens(n, rows, dim):
    import paper_2001_00532_amd as psk
    g = torch.Generator(device="cuda").manual_seed(n)
    ids, dy = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.randn(n, dim, generator=g, device="cuda")
    dE, want = (torch.empty(rows, dim, device="cuda") for _ in range(2))
    ws = psk.psk_embed_grad_workspace(dy, dE)
    psk.psk_embed_grad(ids, dy, dE, padding=3, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        psk.psk_embed_grad(ids, dy, dE, padding=3, ws=ws)
    for _ in range(4):
        ids.copy_(torch.randint(-1, rows, (n,), generator=g, device="cuda", dtype=torch.int32))
        psk.psk_embed_grad(ids, dy, want, padding=3, ws=ws)
        dE.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dE, want)
    R.check(dE, *expected(ids.cpu(), dy.cpu(), rows, 1.0, 3, torch.float32), "replayed")
