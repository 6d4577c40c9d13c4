"""The router and the layer of a mixture of experts against the plain form in 64 bits."""
import math

import numpy as np
import pytest

import serving_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PARTS = {"f16": 2.0 ** -22, "bf16": 2.0 ** -16}


# ------------------------------------------------------------------ router
def routed(x, w, top_k, **kw):
    n = x.shape[0]
    crd = torch.full((n, top_k), 99, dtype=torch.int32, device="cuda")
    vals = torch.full((n, top_k), 99.0, device="cuda")
    psk.psk_moe_route(x.cuda(), w.cuda(), crd, vals, **{k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()})
    return crd.cpu(), vals.cpu()


def compare_route(x, w, top_k, score, bias, normalise, factor, what):
    ids, gates = R.route(x, w, top_k, score, bias, normalise, factor)
    crd, vals = routed(x, w, top_k, score=score, bias=bias, normalise=normalise, factor=factor)
    assert torch.equal(crd, ids), what
    # rounding to 32 bits; the 64-bit logits behind differ by far less
    R.check(vals, gates, gates.abs() * 2.0 ** -23 + 1e-40, what)


@pytest.mark.parametrize("dtype,wtype", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f16", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("n,dim,experts,top_k,score,bias,normalise", [
    (1, 1, 1, 1, 0, False, True), (1, 300, 64, 6, 0, False, True), (9, 77, 65, 8, 1, True, True), (3, 1025, 8, 8, 0, True, False),
    (17, 64, 200, 3, 1, False, False), (2, 40, 1024, 64, 0, False, True)])
def test_route(dtype, wtype, n, dim, experts, top_k, score, bias, normalise):
    rng = np.random.default_rng(n * 100 + experts)
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(TYPES[dtype])
    w = torch.from_numpy(rng.standard_normal((experts, dim)) / math.sqrt(dim)).to(TYPES[wtype])
    b = torch.from_numpy(rng.uniform(-0.3, 0.3, experts)).float() if bias else None
    compare_route(x, w, top_k, score, b, normalise, 1.0 if normalise else 2.5, "%s %s %d experts" % (dtype, wtype, experts))


@pytest.mark.parametrize("score", [0, 1])
def test_equal_logits_go_to_the_lowest_index(score):
    """Equal rows of the router's weights; and logits that differ in the last bits of a long sum only."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((5, 200))).float()
    w = torch.from_numpy(rng.standard_normal((1, 200))).float().repeat(70, 1)
    w[40] = w[40] + 1e-3 * x[2]                              # for token 2 a larger logit
    crd, _ = routed(x, w, 4, score=score)
    assert crd[2].tolist() == [40, 0, 1, 2]
    for t in (0, 1, 3, 4):
        assert crd[t].tolist() in ([0, 1, 2, 3], [40, 0, 1, 2])
    compare_route(x, w, 4, score, None, True, 1.0, "ties")
    big = torch.zeros(1, 200)
    big[0, 0], big[0, 1] = 1.0, 2.0 ** -40
    w = torch.zeros(3, 200)
    w[:, 0] = 1.0
    w[2, 1] = 1.0                                            # larger by 2^-40: invisible in 32 bits
    crd, _ = routed(big, w, 2, score=score)
    assert crd[0].tolist() == [2, 0]


@pytest.mark.parametrize("score", [0, 1])
def test_experts_that_are_never_taken_and_rows_that_are_no_numbers(score):
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((4, 50))).float()
    w = torch.from_numpy(rng.standard_normal((10, 50))).float()
    bias = torch.zeros(10)
    bias[[0, 3, 4, 5, 6, 7, 9]] = -math.inf
    crd, vals = routed(x, w, 6, score=score, bias=bias, normalise=True)
    for t in range(4):
        assert sorted(crd[t, :3].tolist()) == [1, 2, 8] and crd[t, 3:].tolist() == [-1, -1, -1]
        assert vals[t, 3:].tolist() == [0, 0, 0] and abs(float(vals[t].sum()) - 1) < 1e-6
    compare_route(x, w, 6, score, bias, True, 1.0, "few experts")
    bias[:] = -math.inf
    crd, vals = routed(x, w, 6, score=score, bias=bias, normalise=True)
    assert bool((crd == -1).all()) and bool((vals == 0).all())
    x[1, 7] = float("nan")
    crd, vals = routed(x, w, 3, score=score)
    assert crd[1].tolist() == [0, 1, 2] and bool(torch.isnan(vals[1]).all())
    assert bool(torch.isfinite(vals[[0, 2, 3]]).all())
    x[1] = 0
    x[1, 7], w[:, 7] = 1e30, 1e30 * torch.sign(w[:, 7])      # logits of +-1e60
    compare_route(x, w, 3, score, None, False, 1.0, "far logits")


def test_scores_that_underflow():
    x, w = torch.full((2, 1), 1000.0), torch.tensor([[-1.0], [-2.0], [-3.0], [0.0]])
    crd, vals = routed(x, w, 3, score=1, bias=torch.tensor([0.0, 0.0, 0.0, -math.inf]))
    assert crd.tolist() == [[0, 1, 2]] * 2 and vals.tolist() == [[0.0, 0.0, 0.0]] * 2
    crd, vals = routed(x, w, 3, score=0)
    assert crd.tolist() == [[3, 0, 1]] * 2 and vals.tolist() == [[1.0, 0.0, 0.0]] * 2


def test_route_strides():
    rng = np.random.default_rng(5)
    x, w = torch.from_numpy(rng.standard_normal((5, 90))).half(), torch.from_numpy(rng.standard_normal((12, 95))).half()
    a, b = routed(x[:, 3:80].contiguous(), w[:, 5:82].contiguous(), 4)
    xd, wd = x.cuda(), w.cuda()
    crd, vals = torch.empty(5, 4, dtype=torch.int32, device="cuda"), torch.empty(5, 4, device="cuda")
    psk.psk_moe_route(xd[:, 3:80], wd[:, 5:82], crd, vals)
    assert torch.equal(crd.cpu(), a) and torch.equal(vals.cpu(), b)


@pytest.mark.parametrize("experts", [3, 1024])
def test_as_many_tokens_as_a_call_may_have(experts):
    n, dim, top_k = psk.PSK_MAX_VECTORS, 8, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x, w = torch.randn(n, dim, generator=g, device="cuda"), torch.randn(experts, dim, generator=g, device="cuda")
    crd, vals = torch.full((n, top_k), 99, dtype=torch.int32, device="cuda"), torch.full((n, top_k), 99.0, device="cuda")
    psk.psk_moe_route(x, w, crd, vals, normalise=False)
    torch.cuda.synchronize()
    for t in (0, 123457, n - 9):
        ids, gates = R.route(x[t:t + 9].cpu(), w.cpu(), top_k, 0, None, False, 1.0)
        assert torch.equal(crd[t:t + 9].cpu(), ids)
        R.check(vals[t:t + 9], gates, gates.abs() * 2.0 ** -23 + 1e-40, "tokens from %d" % t)


# ------------------------------------------------------------------ layer
def gating(rng, n, experts, top_k, kind="random"):
    crd = np.full((n, top_k), -1, dtype=np.int32)
    for t in range(n):
        k = min(top_k, experts)
        crd[t, :k] = rng.choice(experts, size=k, replace=False)
    if kind == "holes":
        crd[rng.random((n, top_k)) < 0.5] = -1
        crd[n // 2] = -1
        crd[0, 0] = experts                                  # outside: no expert
        crd[n - 1, -1] = -2 ** 31
    elif kind == "none":
        crd[:] = -1
    elif kind == "one":
        crd[:] = -1
        crd[:, top_k // 2] = experts - 1
    elif kind == "twice":
        crd[:] = rng.integers(0, experts, (n, 1))
    return torch.from_numpy(crd), torch.from_numpy(rng.uniform(0.05, 1.0, (n, top_k)).astype(np.float32))


def run16(x, crd, vals, w1, w3, w2, act=0):
    n, dim = x.shape
    buf = torch.full((n + 2, dim + 3), 77.0, dtype=x.dtype, device="cuda")
    y = buf[1:n + 1, :dim]
    psk.psk_moe_experts(x.cuda(), crd.cuda(), vals.cuda(), w1.cuda(), w3.cuda(), w2.cuda(), y, act=act)
    torch.cuda.synchronize()
    assert bool((buf[0] == 77).all()) and bool((buf[n + 1] == 77).all()) and bool((buf[:, dim:] == 77).all()), "wrote past Y"
    return y


def padded(rng, shape, scale, dtype):
    """Weights whose rows are a multiple of 8 apart, NaN behind them."""
    e, r, c = shape
    buf = torch.full((e, r, (c + 7) // 8 * 8 + 8), float("nan"), dtype=dtype)
    buf[:, :, :c] = torch.from_numpy(rng.standard_normal(shape) * scale).to(dtype)
    return buf.cuda()[:, :, :c]


def doubles(w):
    return [m.cpu().double() for m in w]


SHAPES = [(1, 32, 16, 4, 2, "random"), (1, 8, 1, 1, 1, "random"), (3, 100, 45, 5, 3, "holes"), (17, 64, 130, 3, 2, "random"), (6, 200, 72, 70, 8, "random"),
          (40, 72, 24, 2, 2, "random"), (5, 40, 33, 6, 2, "none"), (70, 48, 40, 3, 2, "one"), (9, 520, 260, 4, 4, "twice"), (130, 24, 24, 2, 3, "one")]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,dim,inter,experts,top_k,kind", SHAPES)
def test_layer(dtype, n, dim, inter, experts, top_k, kind):
    t = TYPES[dtype]
    rng = np.random.default_rng(n * 31 + dim)
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
    crd, vals = gating(rng, n, experts, top_k, kind)
    w1, w3 = padded(rng, (experts, inter, dim), 1 / math.sqrt(dim), t), padded(rng, (experts, inter, dim), 1 / math.sqrt(dim), t)
    w2 = padded(rng, (experts, dim, inter), 1 / math.sqrt(inter), t)
    for act in (0, 1):
        ref, bound = R.layer(x, crd, vals, doubles(w1), doubles(w3), doubles(w2), act, t, PARTS[dtype])
        R.check(run16(x, crd, vals, w1, w3, w2, act), ref, bound, "%s act %d %s" % (dtype, act, kind))


def q4_of(w, cols, group):
    return psk.Q4(*(None if t is None else t.cuda() for t in w), cols=cols, group=group)


def q4_doubles(w, cols, group):
    return [R.dequantised(w[0][e], w[1][e], None if w[2] is None else w[2][e], cols, group) for e in range(w[0].shape[0])]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("groups,scale32", [((128, 128), False), ((32, 64), False), ((64, 32), True)])
@pytest.mark.parametrize("n,dim,inter,experts,top_k,kind", SHAPES)
def test_layer_q4(dtype, groups, scale32, n, dim, inter, experts, top_k, kind):
    t = TYPES[dtype]
    st = torch.float32 if scale32 else t
    rng = np.random.default_rng(n * 37 + dim)
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
    crd, vals = gating(rng, n, experts, top_k, kind)
    g1, g2 = groups
    w1 = R.q4_weights(rng, inter, dim, g1, True, st, experts, scale=0.4 / math.sqrt(dim))
    w3 = R.q4_weights(rng, inter, dim, g1, False, st, experts, scale=0.4 / math.sqrt(dim), pad=1)
    w2 = R.q4_weights(rng, dim, inter, g2, True, st, experts, scale=0.4 / math.sqrt(inter))
    y = torch.full((n, dim), 77.0, dtype=t, device="cuda")
    psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), q4_of(w1, dim, g1), q4_of(w3, dim, g1), q4_of(w2, inter, g2), y)
    ref, bound = R.layer(x, crd, vals, q4_doubles(w1, dim, g1), q4_doubles(w3, dim, g1), q4_doubles(w2, inter, g2), 0, t, 2.0 ** -16)
    R.check(y, ref, bound, "q4 %s %s" % (dtype, kind))


LONG = [(5, 1024, 1025, 3, 2, "random"), (20, 1100, 2049, 2, 1, "random"), (6, 2300, 40, 3, 2, "holes"), (18, 72, 4096, 2, 2, "one"),
        (5, 4097, 50, 2, 1, "random"), (7, 40, 4200, 2, 2, "twice"), (4, 2100, 1050, 3, 2, "random"), (37, 700, 530, 2, 1, "random")]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,dim,inter,experts,top_k", [(24, 1500, 200, 8, 4), (65, 2100, 40, 3, 2), (600, 1030, 24, 5, 3), (300, 520, 16, 64, 8)])
def test_many_positions_and_columns(dtype, n, dim, inter, experts, top_k):
    """More positions than a wave looks at, with columns for several workgroups: all see an expert's positions in one order."""
    rng = np.random.default_rng(n)
    t = TYPES[dtype]
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
    crd, vals = gating(rng, n, experts, top_k)
    w = [padded(rng, s, 1 / math.sqrt(s[2]), t) for s in ((experts, inter, dim), (experts, inter, dim), (experts, dim, inter))]
    d = [doubles(m) for m in w]
    ref, bound = R.layer(x, crd, vals, *d, 0, t, PARTS[dtype])
    first = run16(x, crd, vals, *w)
    R.check(first, ref, bound, "16 bits")
    w = [R.q4_weights(rng, r, c, 64, True, t, experts, scale=0.4 / math.sqrt(c)) for r, c in ((inter, dim), (inter, dim), (dim, inter))]
    ref, bound = R.layer(x, crd, vals, *(q4_doubles(m, c, 64) for m, c in zip(w, (dim, dim, inter))), 0, t, 2.0 ** -16)
    A = [q4_of(m, c, 64) for m, c in zip(w, (dim, dim, inter))]
    y = torch.empty(n, dim, dtype=t, device="cuda")
    psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), *A, y)
    R.check(y, ref, bound, "4 bits")
    for _ in range(3):
        again = torch.empty_like(y)
        psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), *A, again)
        assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,dim,inter,experts,top_k,kind", LONG)
def test_long_columns(dtype, n, dim, inter, experts, top_k, kind):
    """Columns on both sides of the lengths at which another kernel or another number of waves takes over."""
    test_layer(dtype, n, dim, inter, experts, top_k, kind)
    test_layer_q4(dtype, (128, 64) if dtype == "f16" else (32, 256), dtype == "bf16", n, dim, inter, experts, top_k, kind)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,top_k,experts,kind", [(4, 3, 3, "twice"), (4, 17, 20, "random"), (4, 64, 3, "twice"), (4, 16, 16, "holes"), (4, 2, 1024, "random"),
                                                  (5, 3, 3, "twice"), (5, 64, 70, "random")])
def test_few_tokens_with_many_entries(dtype, n, top_k, experts, kind):
    """An expert more than four times among four tokens' entries, more than 64 entries, and five tokens beside four."""
    test_layer(dtype, n, 40, 24, experts, top_k, kind)
    test_layer_q4(dtype, (32, 32), False, n, 40, 24, experts, top_k, kind)


def test_matrices_with_groups_and_zero_points_of_their_own():
    """The last matrix has a group of its own, and each of the three zero points or none."""
    rng = np.random.default_rng(16)
    n, dim, inter, experts, t = 6, 300, 150, 4, torch.float16
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
    crd, vals = gating(rng, n, experts, 2)
    for groups, zeros in (((32, 32, 64), (True, False, False)), ((256, 256, 128), (False, True, True)), ((128, 128, 1024), (True, True, False))):
        w = [R.q4_weights(rng, r, c, g, z, t, experts, scale=0.4 / math.sqrt(c))
             for (r, c), g, z in zip(((inter, dim), (inter, dim), (dim, inter)), groups, zeros)]
        y = torch.full((n, dim), 77.0, dtype=t, device="cuda")
        psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), *(q4_of(m, c, g) for m, c, g in zip(w, (dim, dim, inter), groups)), y)
        ref, bound = R.layer(x, crd, vals, *(q4_doubles(m, c, g) for m, c, g in zip(w, (dim, dim, inter), groups)), 0, t, 2.0 ** -16)
        R.check(y, ref, bound, "groups %s" % (groups,))


def test_more_positions_than_one_pair_of_launches_takes():
    """3000 tokens with two experts each: 6000 positions."""
    rng = np.random.default_rng(11)
    n, dim, inter, experts = 3000, 24, 16, 5
    x = torch.from_numpy(rng.standard_normal((n, dim))).bfloat16()
    crd = torch.from_numpy(rng.integers(-1, experts, (n, 2)).astype(np.int32))
    vals = torch.from_numpy(rng.uniform(0.1, 1, (n, 2)).astype(np.float32))
    w = [padded(rng, s, 0.3, torch.bfloat16) for s in ((experts, inter, dim), (experts, inter, dim), (experts, dim, inter))]
    ref, bound = R.layer(x, crd, vals, *map(doubles, w), 0, torch.bfloat16, PARTS["bf16"])
    R.check(run16(x, crd, vals, *w), ref, bound, "6000 positions")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_token_that_is_no_number_spoils_its_own_row(dtype):
    rng = np.random.default_rng(12)
    t, n, dim, inter, experts = TYPES[dtype], 8, 40, 24, 2
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
    crd, vals = gating(rng, n, experts, 2)
    w = [padded(rng, s, 0.2, t) for s in ((experts, inter, dim), (experts, inter, dim), (experts, dim, inter))]
    clean = run16(x, crd, vals, *w).clone()
    x[3, 5], x[6, 39] = float("nan"), float("inf")
    got = run16(x, crd, vals, *w)
    keep = [0, 1, 2, 4, 5, 7]
    assert torch.equal(got[keep], clean[keep])
    assert bool(torch.isnan(got[3]).all()) and not bool(torch.isfinite(got[6]).any())


def test_values_between_the_products_beyond_the_range_of_f16():
    """h of about 10^6 with small weights behind it: Y is an ordinary number."""
    rng = np.random.default_rng(13)
    n, dim, inter = 2, 64, 32
    x = torch.from_numpy(rng.uniform(20, 40, (n, dim))).half()
    w1 = torch.from_numpy(rng.uniform(0.5, 1.0, (1, inter, dim))).half()
    w2 = torch.from_numpy(rng.standard_normal((1, dim, inter)) * 1e-5).half()
    crd, vals = torch.zeros(n, 1, dtype=torch.int32), torch.ones(n, 1)
    ref, bound = R.layer(x, crd, vals, doubles(w1), doubles(w1), doubles(w2), 0, torch.float16, PARTS["f16"])
    R.check(run16(x, crd, vals, w1, w1, w2), ref, bound, "large h")


@pytest.mark.parametrize("n", [3, 9])
def test_small_values_between_the_products(n):
    """h of about 10^-6 with large weights behind it."""
    rng = np.random.default_rng(18)
    dim, inter, t = 64, 200, torch.float16
    x = torch.from_numpy(rng.standard_normal((n, dim)) * 1e-2).half()
    w1 = torch.from_numpy(rng.standard_normal((1, inter, dim)) * 1e-2).half()
    w2 = torch.from_numpy(rng.standard_normal((1, dim, inter)) * 1e3).half()
    crd, vals = torch.zeros(n, 1, dtype=torch.int32), torch.ones(n, 1)
    # the two parts of h are steps of 2^-24 after factors of 2^-8 and 2^11: 2^-24 2^8 2^-11 = 2^-27, half of it the error, which is in the bound
    ref, bound = R.layer(x, crd, vals, doubles(w1), doubles(w1), doubles(w2), 0, t, PARTS["f16"])
    R.check(run16(x, crd, vals, w1, w1, w2), ref, bound, "small h")


def selecting(rows, cols, column, value, dtype, stype=None):
    """One expert's matrix whose rows take `column` (of each row its own where a function) times `value`: 16 bits, and the same in 4
    (scales of type `stype`)."""
    w = torch.zeros(1, rows, cols, dtype=dtype)
    codes = torch.full((1, rows, (cols + 31) // 32 * 16), 0x88, dtype=torch.uint8)
    for r in range(rows):
        c = column(r) if callable(column) else column
        w[0, r, c] = value
        codes[0, r, c // 2] = 0x98 if c % 2 else 0x89       # 9 - 8 = 1 there
    return w, psk.Q4(codes.cuda(), torch.full((1, rows, 1), value, dtype=stype or dtype).cuda(), cols=cols, group=32)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [4, 23])
def test_gelu_keeps_its_relative_error(dtype, n):
    """Pre-activations from -5.5 to 5.5 without any error of their own (one product by 1), the value after them times 2^19 and 2^-6."""
    t, dim = TYPES[dtype], 8
    x = torch.zeros(n, dim, dtype=t)
    x[:, 0], x[:, 1] = torch.linspace(-5.5, 5.5, n).to(t), 1024
    (w1, q1), (w3, q3), (w2, q2) = selecting(dim, dim, 0, 1.0, t), selecting(dim, dim, 1, 512.0, t), selecting(dim, dim, lambda r: r, 2.0 ** -6, t)
    crd, vals = torch.zeros(n, 1, dtype=torch.int32), torch.ones(n, 1)
    ref, _ = R.layer(x, crd, vals, doubles(w1), doubles(w3), doubles(w2), 1, t, 0)
    # of erfc(-v / sqrt 2): two roundings of its argument, times |d log erfc(z) / d log z| <= 2 z^2 + 1 = v^2 + 1; 16 steps for it and three products;
    # rounding of Y (gelu(0) = 0 is its smallest number away at most)
    bound = ref.abs() * (x[:, :1].double() ** 2 + 17) * R.STEP + R.out_error(ref, t)
    R.check(run16(x, crd, vals, w1, w3, w2, 1), ref, bound, "16 bits")
    y = torch.empty(n, dim, dtype=t, device="cuda")
    psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), q1, q3, q2, y, act=psk.PSK_ACT_GELU)
    R.check(y, ref, bound, "4 bits")


@pytest.mark.parametrize("dtype,scale32", [("bf16", False), ("bf16", True), ("f16", True)])
@pytest.mark.parametrize("n", [3, 23])
def test_scales_of_the_layer_near_the_largest_number(dtype, scale32, n):
    """2^-80 in W3, 2^120 in W2 and gates of 2^-40: ordinary numbers before and after."""
    t, dim = TYPES[dtype], 8
    st = torch.float32 if scale32 else t
    x = torch.zeros(n, dim, dtype=t)
    x[:, 0], x[:, 1] = torch.linspace(-3, 3, n).to(t), 1
    q = [selecting(dim, dim, c, v, torch.float32, st)[1] for c, v in ((0, 1.0), (1, 2.0 ** -80), (lambda r: r, 2.0 ** 120))]
    crd, vals = torch.zeros(n, 1, dtype=torch.int32), torch.full((n, 1), 2.0 ** -40)
    ref = R.act(x[:, :1].double(), 0).expand(n, dim)
    y = torch.empty(n, dim, dtype=t, device="cuda")
    psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), *q, y)
    # every sum has one term: 16 steps for the activation and the products, rounding of Y
    R.check(y, ref, ref.abs() * 16 * R.STEP + R.out_error(ref, t), "large scales")


def both_layers(x, pairs, act=0):
    """Y of one expert with 16-bit weights and with 4-bit ones, gate 1; pairs: (16 bits, 4 bits) of W1, W3, W2."""
    n, dim = x.shape
    crd, vals = torch.zeros(n, 1, dtype=torch.int32), torch.ones(n, 1)
    y = torch.empty(n, dim, dtype=x.dtype, device="cuda")
    psk.psk_moe_experts_q4(x.cuda(), crd.cuda(), vals.cuda(), *(q for _, q in pairs), y, act=act)
    return ("16 bits", run16(x, crd, vals, *(w for w, _ in pairs), act)), ("4 bits", y)


def ones(rows, cols, at, dtype):
    """One expert's matrix of 1 and -1 at places (row, column, sign), 0 elsewhere: 16 bits, and the same in 4."""
    w, codes = torch.zeros(1, rows, cols, dtype=dtype), torch.full((1, rows, (cols + 31) // 32 * 16), 0x88, dtype=torch.uint8)
    for r, c, sign in at:
        w[0, r, c] = sign
        codes[0, r, c // 2] += sign * (16 if c % 2 else 1)
    return w, psk.Q4(codes.cuda(), torch.ones(1, rows, 1, dtype=dtype).cuda(), cols=cols, group=8192)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 23])
@pytest.mark.parametrize("x1,w3,w2", [(-10, -14, 15), (10, 15, -14)])
def test_far_values_between_the_products_keep_their_relative_error(dtype, n, x1, w3, w2):
    """h of about 2^-24 and of about 2^25, every sum of one term."""
    t, dim = TYPES[dtype], 8
    x = torch.zeros(n, dim, dtype=t)
    x[:, 0], x[:, 1] = torch.linspace(0.7, 3, n).to(t), 2.0 ** x1
    pairs = selecting(dim, dim, 0, 1.0, t), selecting(dim, dim, 1, 2.0 ** w3, t), selecting(dim, dim, lambda r: r, 2.0 ** w2, t)
    ref = (R.act(x[:, :1].double(), 0) * 2.0 ** (x1 + w3 + w2)).expand(n, dim)
    for what, y in both_layers(x, pairs):
        # 16 steps of 32 bits for the activation and the products
        R.check(y, ref, ref.abs() * 16 * R.STEP + R.out_error(ref, t), what)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 23])
@pytest.mark.parametrize("inter", [8, 1500, 3000, 4104])
def test_values_between_the_products_keep_32_bits(dtype, n, inter):
    """Differences of two h that agree in their first 11 to 13 bits: h[2i] = s (1 + d), h[2i+1] = s with s = silu(v), Y = s d.  Every way of the
    second product, by its columns."""
    t, dim = TYPES[dtype], 8
    rng = np.random.default_rng(n)
    x = torch.zeros(n, dim, dtype=t)
    x[:, 0], x[:, 1], x[:, 2] = torch.linspace(0.7, 3, n).to(t), 1, torch.from_numpy(2.0 ** rng.uniform(-13, -11, n)).to(t)
    pairs = (ones(inter, dim, [(r, 0, 1) for r in range(inter)], t), ones(inter, dim, [(r, 1, 1) for r in range(inter)] + [(r, 2, 1) for r in range(0, inter, 2)], t),
             ones(dim, inter, [(r, 2 * (r * (inter // 2 - 1) // 7) + k, 1 - 2 * k) for r in range(dim) for k in (0, 1)], t))
    s = R.act(x[:, :1].double(), 0)
    ref = (s * x[:, 2:3].double()).expand(n, dim)
    # s is the same number in both: its 16 steps count relative to Y.  1 + d in 32 bits and the product with it: half a step each, in both; the second
    # product adds up six parts of at most s (1 + d) each: a step of the sizes so far, of 2 s, for each
    bound = ref.abs() * 16 * R.STEP + s.abs() * (2 + 6 * 2) * 1.001 * R.STEP + R.out_error(ref, t)
    for what, y in both_layers(x, pairs):
        R.check(y, ref, bound, what)


@pytest.mark.parametrize("n", [1, 3, 23])
def test_infinite_values_between_the_products(n):
    """h beyond 2^128 in every other token: Y is infinite there (all weights behind h are 1) and finite in the others."""
    dim = 8
    x = torch.zeros(n, dim, dtype=torch.bfloat16)
    x[:, 0], x[:, 1] = torch.linspace(0.7, 3, n).to(torch.bfloat16), 2.0 ** -70
    x[0::2, 1] = 2.0 ** 70
    pairs = (selecting(dim, dim, 0, 1.0, torch.bfloat16), selecting(dim, dim, 1, 2.0 ** 60, torch.bfloat16),
             ones(dim, dim, [(r, c, 1) for r in range(dim) for c in range(dim)], torch.bfloat16))
    ref = (8 * R.act(x[:, :1].double(), 0) * x[:, 1:2].double() * 2.0 ** 60).expand(n, dim).clone()
    ref[0::2] = math.inf
    for what, y in both_layers(x, pairs):
        R.check(y, ref, ref.abs() * 32 * R.STEP + R.out_error(ref, torch.bfloat16), what)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("top_k,experts", [(5, 3), (3, 1), (64, 2), (20, 30)])
def test_one_token_with_an_expert_in_every_slot(dtype, top_k, experts):
    test_layer(dtype, 1, 72, 40, experts, top_k, "twice")
    test_layer_q4(dtype, (32, 64), False, 1, 72, 40, experts, top_k, "twice")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,dim,inter", [(1, 1231, 311), (3, 77, 129), (9, 1231, 311), (50, 333, 45), (7, 9, 3)])
def test_weights_at_any_element(dtype, n, dim, inter):
    """Rows of weights that begin at odd elements, NaN around them; and weights without any padding, up to the end of their tensor."""
    t, experts, top_k = TYPES[dtype], 5, 2
    rng = np.random.default_rng(dim)
    x = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
    crd, vals = gating(rng, n, experts, top_k)

    def loose(shape):
        e, r, c = shape
        buf = torch.full((e, r + 1, c + 3), float("nan"), dtype=t)
        buf[:, 1:, 3:] = torch.from_numpy(rng.standard_normal(shape) / math.sqrt(c)).to(t)
        return buf.cuda()[:, 1:, 3:]
    w = [loose(s) for s in ((experts, inter, dim), (experts, inter, dim), (experts, dim, inter))]
    ref, bound = R.layer(x, crd, vals, *map(doubles, w), 0, t, PARTS[dtype])
    got = run16(x, crd, vals, *w)
    R.check(got, ref, bound, "odd strides")
    assert torch.equal(got, run16(x, crd, vals, *(m.contiguous() for m in w)))


@pytest.mark.parametrize("n", [1, 5])
@pytest.mark.parametrize("dim,inter", [((1 << 28) - 256, 16), (16, (1 << 28) - 256)])
def test_as_many_rows_and_columns_as_a_matrix_may_have(n, dim, inter):
    """Weights that are zero but in the first and the last two columns, 16 bits and 4."""
    t = torch.bfloat16
    crd, vals = torch.zeros(n, 1, dtype=torch.int32, device="cuda"), torch.ones(n, 1, device="cuda")
    x = torch.zeros(n, dim, dtype=t, device="cuda")
    x[:, 0], x[:, -2], x[:, -1] = (torch.linspace(a, b, n) for a, b in ((0.5, 1), (-1, 2), (1, -0.5)))
    # a = u = x[0] + x[-2] - x[-1], Y = h[0] + h[-2] - h[-1] with h alike in all columns
    v = x[:, 0].double() + x[:, -2].double() - x[:, -1].double()
    size = x[:, 0].double().abs() + x[:, -2].double().abs() + x[:, -1].double().abs()
    h = R.act(v, 0) * v
    # sums of three numbers (and zeros): 8 steps of their sizes in a and in u, |act'| <= 1.13; 16 steps for the activation and the products; Y is three h
    bound = 3 * ((1.13 + 1) * 8 * R.STEP * size * (v.abs() + size) + 24 * R.STEP * h.abs()) + R.out_error(h, t)

    def wide(rows, cols):
        w = torch.zeros(1, rows, cols, dtype=t, device="cuda")
        w[:, :, 0], w[:, :, -2], w[:, :, -1] = 1, 1, -1
        return w

    def four(rows, cols):
        codes = torch.full((1, rows, cols // 32 * 16 + 16), 0x88, dtype=torch.uint8, device="cuda")
        codes[:, :, 0] = 0x89
        codes[:, :, cols // 2 - 1] = 0x79
        return psk.Q4(codes, torch.ones(1, rows, 1, dtype=t, device="cuda"), cols=cols, group=1 << 30)
    for make, call in ((wide, psk.psk_moe_experts), (four, psk.psk_moe_experts_q4)):
        y = torch.full((n, dim), 77.0, dtype=t, device="cuda")
        call(x, crd, vals, make(inter, dim), make(inter, dim), make(dim, inter), y)
        torch.cuda.synchronize()
        off = (y.double() - h[:, None]).abs() / bound[:, None]
        assert float(off.max()) <= 1, float(off.max())


def test_one_matrix_holds_both_halves():
    """W1 and W3 as the halves of one tensor, experts a stride apart."""
    rng = np.random.default_rng(14)
    n, dim, inter, experts = 4, 48, 32, 3
    both = torch.from_numpy(rng.standard_normal((experts, 2 * inter, dim)) * 0.2).bfloat16().cuda()
    w2 = torch.from_numpy(rng.standard_normal((experts, dim, inter)) * 0.2).bfloat16().cuda()
    x = torch.from_numpy(rng.standard_normal((n, dim))).bfloat16()
    crd, vals = gating(rng, n, experts, 2)
    a = run16(x, crd, vals, both[:, :inter], both[:, inter:], w2)
    b = run16(x, crd, vals, both[:, :inter].contiguous(), both[:, inter:].contiguous(), w2)
    assert torch.equal(a, b)


@pytest.mark.parametrize("n", [2, 9])
def test_two_calls_at_once(n):
    """Two streams, a workspace each: what both give alone."""
    rng = np.random.default_rng(17)
    dim, inter, experts, t = 1100, 600, 6, torch.bfloat16
    w = [torch.from_numpy(rng.standard_normal(s) * 0.05).to(t).cuda() for s in ((experts, inter, dim), (experts, inter, dim), (experts, dim, inter))]
    calls = []
    for _ in range(2):
        x = torch.from_numpy(rng.standard_normal((n, dim))).to(t).cuda()
        crd, vals = (v.cuda() for v in gating(rng, n, experts, 2))
        calls.append((x, crd, vals, torch.empty_like(x), torch.empty_like(x), psk.psk_moe_workspace(n, dim, inter, experts, 2), torch.cuda.Stream()))
    for x, crd, vals, alone, _, ws, _ in calls:
        psk.psk_moe_experts(x, crd, vals, *w, alone, ws=ws)
    torch.cuda.synchronize()
    for _ in range(20):
        for x, crd, vals, _, y, ws, stream in calls:
            psk.psk_moe_experts(x, crd, vals, *w, y, ws=ws, stream=stream)
    torch.cuda.synchronize()
    for _, _, _, alone, y, _, _ in calls:
        assert torch.equal(alone, y)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_serving_step(dtype):
    """A projection in 4 bits, the router on what it gives and the layer in 4 bits, eager on a side stream and captured; every
    replay follows new activations and another number of padded tokens, with eager work in between."""
    t = TYPES[dtype]
    rng = np.random.default_rng(15)
    n, dim, inter, experts, top_k, group = 5, 256, 96, 12, 3, 64
    wp = R.q4_weights(rng, dim, dim, group, True, t, scale=0.5 / math.sqrt(dim))
    w1, w3 = (R.q4_weights(rng, inter, dim, group, True, t, experts, scale=0.4 / math.sqrt(dim)) for _ in range(2))
    w2 = R.q4_weights(rng, dim, inter, group, True, t, experts, scale=0.4 / math.sqrt(inter))
    wr = torch.from_numpy(rng.standard_normal((experts, dim)) / math.sqrt(dim)).to(t)
    P, A1, A3, A2, wrd = q4_of(wp, dim, group), q4_of(w1, dim, group), q4_of(w3, dim, group), q4_of(w2, inter, group), wr.cuda()
    x, z, y = (torch.zeros(n, dim, dtype=t, device="cuda") for _ in range(3))
    crd, vals = torch.zeros(n, top_k, dtype=torch.int32, device="cuda"), torch.zeros(n, top_k, device="cuda")
    ws = (psk.psk_gemm_q4_workspace(P, x), psk.psk_moe_route_workspace(n, experts), psk.psk_moe_workspace(n, dim, inter, experts, top_k))

    def step():
        psk.psk_gemm_q4(P, x, z, ws=ws[0])
        psk.psk_moe_route(z, wrd, crd, vals, ws=ws[1])
        psk.psk_moe_experts_q4(z, crd, vals, A1, A3, A2, y, ws=ws[2])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    dense = q4_doubles(w1, dim, group), q4_doubles(w3, dim, group), q4_doubles(w2, inter, group)
    for rep in range(4):
        xh = torch.from_numpy(rng.standard_normal((n, dim))).to(t)
        x.copy_(xh)
        for b in ws:
            b.fill_(0xFF)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        ref, bound = R.gemm(R.dequantised(*wp, dim, group), xh, t)
        R.check(z, ref, bound, "projection %d" % rep)
        ids, gates = R.route(z.cpu(), wr, top_k, 0, None, True, 1.0)
        assert torch.equal(crd.cpu(), ids)
        R.check(vals, gates, gates.abs() * 2.0 ** -23 + 1e-40, "gates %d" % rep)
        ref, bound = R.layer(z.cpu(), crd.cpu(), vals.cpu(), *dense, 0, t, 2.0 ** -16)
        R.check(y, ref, bound, "layer %d" % rep)
        kept = y.clone()
        step()
        assert torch.equal(kept, y)
