"""The embedding lookup and its gradient against the plain form in 64 bits."""
import numpy as np
import pytest

import ends_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def ints(v):
    return torch.as_tensor(v, dtype=torch.int32)


def tokens(rng, n, rows, kind):
    if kind == "uniform":
        return ints(rng.integers(0, rows, n))
    if kind == "one":
        return torch.full((n,), rows - 1, dtype=torch.int32)
    if kind == "none":
        return ints(rng.choice([-1, rows, 2 ** 31 - 1, -2 ** 31], n))
    if kind == "head":                                      # most of them one token, some holes
        return ints(np.where(rng.random(n) < 0.7, rows // 2, rng.integers(-2, rows + 2, n)))
    return ints(np.minimum(rng.zipf(1.3, n) - 1, rows))     # "zipf": some fall behind the last row


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("table", ["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (5, 3, 7), (9, 4, 8), (70, 10, 9), (3, 20, 63), (200, 50, 64), (33, 7, 100), (17, 30, 515), (2, 9, 2048), (6, 5, 4101)])
def test_embed(dtype, table, n, rows, dim):
    rng = np.random.default_rng(n * 31 + dim)
    ids, factor = tokens(rng, n, rows, "head" if n > 8 else "uniform"), (1.0 if n % 2 else 7.3)
    wide = torch.full((n + 1, dim + 3), 77.0, dtype=TYPES[dtype], device="cuda")
    Y = wide[:n, 1:1 + dim]
    if table == "i8":
        codes, scales = torch.from_numpy(rng.integers(-128, 128, (rows, (dim + 15) // 16 * 16 + 16), dtype=np.int8)), torch.rand(rows) / 100
        psk.psk_embed(ids.cuda(), psk.I8(codes.cuda(), scales.cuda(), cols=dim), Y, factor=factor)
        ref, bound = R.embed(ids, codes[:, :dim], float(np.float32(factor)), TYPES[dtype], scales)
    else:
        E = torch.full((rows, dim + 5), float("nan"), dtype=TYPES[table])
        E[:, 3:3 + dim] = torch.from_numpy(rng.standard_normal((rows, dim))).to(TYPES[table])
        psk.psk_embed(ids.cuda(), E.cuda()[:, 3:3 + dim], Y, factor=factor)
        ref, bound = R.embed(ids, E[:, 3:3 + dim], float(np.float32(factor)), TYPES[dtype])
    R.check(Y, ref, bound, "embed %s %s" % (table, dtype))
    assert bool((wide[:, 0] == 77).all()) and bool((wide[:, 1 + dim:] == 77).all()) and bool((wide[n] == 77).all())


def test_embed_without_rows_or_tokens():
    Y = torch.full((3, 20), 77.0, device="cuda")
    psk.psk_embed(ints([0, 1, -1]).cuda(), torch.empty((0, 20), device="cuda"), Y)
    assert bool((Y == 0).all())
    psk.psk_embed(ints([0, 1, -1]).cuda(), psk.I8(torch.empty((0, 32), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), cols=20), Y)
    assert bool((Y == 0).all())
    psk.psk_embed(ints([]).cuda(), torch.ones((4, 20), device="cuda"), Y[:0])
    psk.psk_embed(ints([1]).cuda(), torch.ones((4, 0), device="cuda"), Y[:1, :0])


def test_embed_keeps_what_a_row_holds():
    """Infinities and NaN of a row that a token has; not those of row 0 for a token that is none."""
    E = torch.zeros(4, 16)
    E[0], E[2, 3], E[2, 4] = float("nan"), float("inf"), float("nan")
    Y = torch.empty(3, 16, device="cuda")
    psk.psk_embed(ints([-1, 2, 9]).cuda(), E.cuda(), Y, factor=2.0)
    assert bool((Y[0] == 0).all()) and bool((Y[2] == 0).all()) and float(Y[1, 3]) == float("inf") and bool(torch.isnan(Y[1, 4])) and float(Y[1, 5]) == 0


def test_embed_past_32_bits():
    """A table and a result of more than 2^32 bytes."""
    rows, dim = 2200, 1 << 20
    E = torch.zeros((rows, dim), dtype=torch.float16, device="cuda")             # 4.6 GB
    E[rows - 1], E[1] = 3, 2
    ids = torch.full((2049,), 1, dtype=torch.int32, device="cuda")
    ids[2048] = rows - 1
    Y = torch.empty((2049, dim), dtype=torch.float16, device="cuda")
    psk.psk_embed(ids, E, Y)
    assert bool((Y[2048] == 3).all()) and bool((Y[:2048:73] == 2).all())
    psk.psk_embed_grad(ids, Y, E)
    assert bool((E[rows - 1] == 3).all()) and bool((E[1] == 2 * 2048).all()) and bool((E[0] == 0).all()) and bool((E[2:rows - 1:61] == 0).all())


@pytest.mark.parametrize("table,dtype", [("f32", "f32"), ("i8", "f32"), ("f16", "bf16")])
def test_results_larger_than_the_caches(table, dtype):
    """From 32 MB on they are stored past them: rows at odd places, a last piece that is the row's last; and the gradient."""
    test_embed(dtype, table, 5999, 40, 3001)
    if dtype == "f32":
        rng = np.random.default_rng(1)
        ids, dy = tokens(rng, 900, 4001, "zipf"), torch.from_numpy(rng.standard_normal((900, 2101))).to(TYPES["bf16" if table == "i8" else "f32"])
        for m in (900, 60):
            ref, bound = R.embed_grad(ids[:m], dy[:m], 4001, 1.0, -1, torch.float32)
            R.check(gradient(ids[:m], dy[:m], 4001, "f32"), ref, bound, "large gradient")


# ------------------------------------------------------------------ the gradient
def gradient(ids, dy, rows, gtype, factor=1.0, padding=-1, old=None, pad=3):
    n, dim = dy.shape
    wide = torch.full((rows + 2, dim + pad), 77.0, dtype=TYPES[gtype], device="cuda")
    dE = wide[1:rows + 1, 1:1 + dim]
    if old is not None:
        dE.copy_(old)
    src = torch.full((n, dim + 5), float("nan"), dtype=dy.dtype)
    src[:, 2:2 + dim] = dy
    ws = torch.full((psk.psk_embed_grad_workspace_bytes(n, rows, dim),), 0xa5, dtype=torch.uint8, device="cuda")
    psk.psk_embed_grad(ids.cuda(), src.cuda()[:, 2:2 + dim], dE, factor=factor, padding=padding, accumulate=old is not None, ws=ws)
    torch.cuda.synchronize()
    assert bool((wide[0] == 77).all()) and bool((wide[rows + 1] == 77).all()) and bool((wide[:, 0] == 77).all()) and bool((wide[:, 1 + dim:] == 77).all())
    return dE


@pytest.mark.parametrize("dtype,gtype", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("kind", ["uniform", "one", "none", "head", "zipf"])
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (2, 5, 7), (63, 300, 8), (64, 20, 9), (65, 33, 20), (130, 1, 64), (700, 70, 100), (1025, 520, 31), (2049, 2000, 72),
                                        (300, 40, 515), (257, 30, 1027), (5000, 700, 16)])
def test_gradient(dtype, gtype, kind, n, rows, dim):
    rng = np.random.default_rng(n * 13 + rows + dim)
    ids, dy = tokens(rng, n, rows, kind), torch.from_numpy(rng.standard_normal((n, dim))).to(TYPES[dtype])
    ref, bound = R.embed_grad(ids, dy, rows, 1.0, -1, TYPES[gtype])
    R.check(gradient(ids, dy, rows, gtype), ref, bound, "gradient %s %s" % (kind, dtype))


@pytest.mark.parametrize("dtype,gtype", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("n,rows,dim", [(3, 4, 5), (40, 9, 12), (500, 60, 77), (1500, 3, 600), (4500, 900, 24)])
def test_gradient_added_scaled_and_padded(dtype, gtype, n, rows, dim):
    rng = np.random.default_rng(n + rows)
    ids, dy = tokens(rng, n, rows, "head"), torch.from_numpy(rng.standard_normal((n, dim))).to(TYPES[dtype])
    old = torch.from_numpy(rng.standard_normal((rows, dim))).to(TYPES[gtype])
    factor = float(np.float32(dim ** 0.5))
    for padding in (-1, rows // 2, 0):
        ref, bound = R.embed_grad(ids, dy, rows, factor, padding, TYPES[gtype], old)
        R.check(gradient(ids, dy, rows, gtype, factor, padding, old), ref, bound, "added, padding %d" % padding)
        ref, bound = R.embed_grad(ids, dy, rows, factor, padding, TYPES[gtype])
        R.check(gradient(ids, dy, rows, gtype, factor, padding), ref, bound, "assigned, padding %d" % padding)


@pytest.mark.parametrize("n,rows", [(33000, 200001), (70001, 300), (16385, 600000), (4097, 1 << 25)])
def test_gradient_of_many_tokens(n, rows):
    """More than one workgroup sorts, two to three digits; a row of thousands of tokens among rows of one."""
    rng = np.random.default_rng(n)
    ids, dy = tokens(rng, n, min(rows, 200001), "head"), torch.from_numpy(rng.standard_normal((n, 3))).float()
    if rows == 1 << 25:
        ids[::7] = torch.from_numpy(rng.integers(0, rows, ids[::7].numel())).int()
    used = torch.unique(ids[(ids >= 0) & (ids < rows)].long())
    got = gradient(ids, dy, rows, "f32")
    place = {v: i for i, v in enumerate(used.tolist())}
    ref, bound = R.embed_grad(ints([place.get(v, -1) for v in ids.tolist()]), dy, used.numel(), 1.0, -1, torch.float32)
    R.check(got[used.cuda()], ref, bound, "many tokens")
    assert int((got != 0).any(1).sum()) <= used.numel()


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2048, 2049, 65535, 65536, 65537])
def test_gradient_where_the_way_changes(n):
    """One launch, ranges of rows, several workgroups that sort; padding that is a row among the others; tokens of the last rows."""
    rng = np.random.default_rng(n)
    for rows, dim in ((300, 20), (1000, 5)):
        ids, dy = tokens(rng, n, rows, "head"), torch.from_numpy(rng.standard_normal((n, dim))).half()
        ids[-1] = 2
        for padding in (2, rows - 1):
            ref, bound = R.embed_grad(ids, dy, rows, 1.0, padding, torch.float32)
            R.check(gradient(ids, dy, rows, "f32", padding=padding), ref, bound, "%d tokens, padding %d" % (n, padding))


def test_gradient_of_one_row_among_very_many():
    """More than 524288 rows with few tokens and with many; one row's tokens over hundreds of tiles."""
    for n, rows in ((700, 524288), (700, 524289), (3000, 524289), (1, 3_000_000)):
        ids = torch.full((n,), rows - 1, dtype=torch.int32)
        ids[n // 2:n // 2 + 1] = 0
        dy = torch.ones(n, 4)
        got = gradient(ids, dy, rows, "f32", pad=5)
        assert bool((got[rows - 1] == n - 1).all()) and bool((got[0] == 1).all()) and float(got.sum()) == 4 * n


def test_gradient_without_tokens_or_rows():
    dE = torch.full((7, 20), 77.0, device="cuda")
    none = ints([]).cuda()
    psk.psk_embed_grad(none, torch.empty((0, 20), device="cuda"), dE, accumulate=True)
    assert bool((dE == 77).all())
    psk.psk_embed_grad(none, torch.empty((0, 20), device="cuda"), dE)
    assert bool((dE == 0).all())
    psk.psk_embed_grad(ints([0, 1]).cuda(), torch.ones((2, 20), device="cuda"), dE[:0])


def test_gradient_keeps_infinities_to_their_rows():
    """A token's NaN reaches its own row only, also where it is the neighbour in a tile, and not at all if the token is padding."""
    n, rows, dim = 200, 50, 40
    rng = np.random.default_rng(2)
    ids, dy = tokens(rng, n, rows, "uniform"), torch.from_numpy(rng.standard_normal((n, dim))).float()
    ids[3], ids[100], ids[150] = 11, 12, -1
    dy[3, 5], dy[100, 7], dy[150], dy[ids == 20] = float("nan"), float("inf"), float("nan"), float("nan")
    ref, bound = R.embed_grad(ids, dy, rows, 1.0, 20, torch.float32)
    R.check(gradient(ids, dy, rows, "f32", padding=20), ref, torch.nan_to_num(bound, nan=1.0, posinf=1.0), "not finite")


def test_gradient_against_differences():
    """The lookup is linear in the table: (loss(E + h) - loss(E - h)) / 2h = the gradient, loss = sum of Y * dY."""
    rng = np.random.default_rng(5)
    n, rows, dim = 90, 12, 17
    ids, dy, E = tokens(rng, n, rows, "head"), torch.from_numpy(rng.standard_normal((n, dim))).float(), torch.from_numpy(rng.standard_normal((rows, dim))).float()
    got = gradient(ids, dy, rows, "f32", factor=1.5).cpu().double()

    def loss(table):
        Y = torch.empty((n, dim), device="cuda")
        psk.psk_embed(ids.cuda(), table.cuda(), Y, factor=1.5)
        return float((Y.cpu().double() * dy.double()).sum())
    for v, j in ((0, 0), (rows // 2, 3), (rows - 1, dim - 1), (5, 9)):
        h, up, down = 0.5, E.clone(), E.clone()
        up[v, j] += h
        down[v, j] -= h
        step = float(up[v, j]) - float(down[v, j])
        size = float((dy[:, j].double().abs() * (ids == v)).sum()) * 1.5
        # each value of Y is rounded once (|Y| < 8), each sum of the gradient (n + 2) times at most
        assert abs((loss(up) - loss(down)) / step - float(got[v, j])) <= size * (n + 2) * R.ULP + 2 * 8 * R.ULP / step * float(dy[:, j].abs().sum()) + 1e-12


def test_gradient_twice_the_same_bits():
    rng = np.random.default_rng(6)
    for n, rows, dim in ((3000, 50, 100), (40000, 5000, 24)):
        ids, dy = tokens(rng, n, rows, "zipf"), torch.from_numpy(rng.standard_normal((n, dim))).float()
        assert torch.equal(gradient(ids, dy, rows, "f32"), gradient(ids, dy, rows, "f32"))
