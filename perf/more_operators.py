"""Operators at the two ends of a language model, and its projections in 8 bits, as they are measured: the embedding lookup with
scaling, its gradient by sorted tokens, and the products of 8-bit integers with scales for each token and channel, from
activations that are quantised in the call (linear) and from codes that a program has already (gemm).

Every case is one call with its sizes.  prepare() makes what a program holds: tokens, tables, weights, output buffers and
workspaces.  With `own` false run() computes the plain form with elementary torch operations in 32 bits (the codes of activations
in 64: a value next to a border between two codes).
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # a step of 32 sequences decoded together, from a table in 8 bits that the output layer shares: launch latency counts
        {"name": "embed_step", "op": "embed", "n": 32, "vocab": 32768, "dim": 4096, "table": "i8", "dtype": "bf16", "scaled": False, "holes": 0.0},
        # a long prompt, a large vocabulary, rows times sqrt(dim)
        {"name": "embed_prompt", "op": "embed", "n": 16384, "vocab": 131072, "dim": 4096, "table": "bf16", "dtype": "bf16", "scaled": True, "holes": 0.0},
        # a ragged batch with padding, a table kept in 32 bits, rows that fill no line of memory
        {"name": "embed_odd", "op": "embed", "n": 5003, "vocab": 50001, "dim": 1027, "table": "f32", "dtype": "f16", "scaled": True, "holes": 0.1},
        # the gradient of a small model's step
        {"name": "grad_small", "op": "grad", "n": 512, "vocab": 8192, "dim": 1024, "dtype": "f32", "gtype": "f32", "scaled": False, "holes": 0.0, "head": 0.0},
        # four sequences of 4096 tokens, gradient in 32 bits
        {"name": "grad_train", "op": "grad", "n": 16384, "vocab": 32768, "dim": 4096, "dtype": "bf16", "gtype": "f32", "scaled": True, "holes": 0.0, "head": 0.0},
        # more tokens than a workgroup sorts, a third of them one token, odd rows, some without a token
        {"name": "grad_pad", "op": "grad", "n": 40001, "vocab": 50001, "dim": 1027, "dtype": "f16", "gtype": "f16", "scaled": False, "holes": 0.1, "head": 0.33},
        # a projection for one token: launch latency counts
        {"name": "i8_mv", "op": "linear", "rows": 4096, "cols": 4096, "n": 1, "dtype": "bf16", "bias": True},
        # the output layer over a vocabulary, one token
        {"name": "i8_mv_large", "op": "linear", "rows": 32768, "cols": 8192, "n": 1, "dtype": "bf16", "bias": False},
        # 32 sequences decoded together
        {"name": "i8_mm_batch", "op": "linear", "rows": 10240, "cols": 4096, "n": 32, "dtype": "f16", "bias": False},
        # a prompt through a projection, quantised on the way
        {"name": "i8_mm_prompt", "op": "linear", "rows": 8192, "cols": 4096, "n": 2048, "dtype": "bf16", "bias": True},
        # sizes that fill no tile, results in 32 bits
        {"name": "i8_codes_odd", "op": "gemm", "rows": 5003, "cols": 2051, "n": 333, "dtype": "f32", "bias": True},
        # several prompts, codes at hand because an earlier projection of the same activations made them
        {"name": "i8_codes_large", "op": "gemm", "rows": 16384, "cols": 4096, "n": 8192, "dtype": "bf16", "bias": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "grad", "grad", "linear", "linear", "gemm"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("embed", "grad"):
        n, vocab = _log(rng, 1, 40000), _log(rng, 1000, 131072)
        dim = _log(rng, 64, min(8192, 65_000_000 // max(n, vocab)))
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        c = {"op": op, "n": n, "vocab": vocab, "dim": dim, "dtype": dtype, "scaled": rng.random() < 0.5, "holes": rng.choice([0.0, 0.0, 0.1, 0.5])}
        if op == "embed":
            return dict(c, table=rng.choice(["f32", "i8", "bf16", "f16"]))
        return dict(c, gtype=rng.choice(["f32", dtype]), head=rng.choice([0.0, 0.0, 0.3, 0.9]))
    n = rng.choice([1, 1, rng.randint(2, 16), rng.randint(17, 128), _log(rng, 129, 8192), _log(rng, 129, 8192)])
    cols = _log(rng, 256, 16384)
    rows = _log(rng, 256, min(32768, 260_000_000 // cols, 270_000_000_000 // cols // n))
    if rng.random() < 0.5:
        rows, cols = (rows + 63) // 64 * 64, (cols + 127) // 128 * 128
    return {"op": op, "rows": rows, "cols": cols, "n": n, "dtype": dtype, "bias": rng.random() < 0.5}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + 31)
    return g


def _chances(vocab, device):
    """How often each token occurs: about one over its place in the order of frequency."""
    p = 1.0 / (torch.arange(vocab, dtype=torch.float64, device=device) + 2.7)
    return p / p.sum()


def _tokens(case, g):
    """Tokens of text; a share `head` of them is one token, a share `holes` of the places holds none (-1)."""
    n, vocab = case["n"], case["vocab"]
    place = torch.searchsorted(torch.cumsum(_chances(vocab, "cuda"), 0), torch.rand(n, generator=g, device="cuda", dtype=torch.float64))
    order = torch.randperm(vocab, generator=g, device="cuda")
    ids = order[place.clamp(max=vocab - 1)]
    u = torch.rand(n, generator=g, device="cuda")
    ids = torch.where(u < case.get("head", 0.0), order[:1], ids)
    return torch.where(torch.rand(n, generator=g, device="cuda") < case["holes"], -1, ids).to(torch.int32)


def _activations(n, dim, dtype, g):
    """About normal, one feature in a hundred ten times as large (as the residual stream of a trained model has)."""
    x = torch.randn((n, dim), generator=g, device="cuda")
    big = torch.rand((1, dim), generator=g, device="cuda") < 0.01
    return torch.where(big, 10 * x, x).to(TYPES[dtype])


def _codes(n, cols, g):
    """n x cols codes, each row in a multiple of 16 bytes."""
    c = torch.empty((n, (cols + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    for r in range(0, n, 4096):
        part = c[r:r + 4096]
        part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 31).round().clamp(-127, 127))
    return c


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = {"case": case, "factor": math.sqrt(case["dim"]) if case.get("scaled") else 1.0}
    if op == "embed":
        s["ids"] = _tokens(case, g)
        if case["table"] == "i8":
            s["codes"] = _codes(case["vocab"], case["dim"], g)
            s["scales"] = (0.5 + torch.rand(case["vocab"], generator=g, device="cuda")) / 1000
        else:
            s["table"] = (torch.randn((case["vocab"], case["dim"]), generator=g, device="cuda") * 0.03).to(TYPES[case["table"]])
    elif op == "grad":
        s["ids"] = _tokens(case, g)
        s["dy"] = (torch.randn((case["n"], case["dim"]), generator=g, device="cuda") * 0.01).to(TYPES[case["dtype"]])
    else:
        rows, cols, n = case["rows"], case["cols"], case["n"]
        s["codes"] = _codes(rows, cols, g)
        s["scales"] = (0.5 + torch.rand(rows, generator=g, device="cuda")) / (31 * math.sqrt(cols))
        s["bias"] = torch.randn(rows, generator=g, device="cuda") if case["bias"] else None
        if op == "linear":
            s["x"] = _activations(n, cols, case["dtype"], g)
        else:
            s["xcodes"] = _codes(n, cols, g)
            s["xscales"] = (0.5 + torch.rand(n, generator=g, device="cuda")) / 31
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program of the framework keeps beside the tensors: descriptions of 8-bit matrices, outputs, workspaces."""
    import paper_2001_00532_amd as psk

    case = s["case"]
    op, n = case["op"], case["n"]
    s["psk"] = psk
    if op == "embed":
        s["E"] = psk.I8(s["codes"], s["scales"], cols=case["dim"]) if case["table"] == "i8" else s["table"]
        s["y"] = torch.empty((n, case["dim"]), dtype=TYPES[case["dtype"]], device="cuda")
    elif op == "grad":
        s["de"] = torch.empty((case["vocab"], case["dim"]), dtype=TYPES[case["gtype"]], device="cuda")
        s["ws"] = psk.psk_embed_grad_workspace(s["dy"], s["de"])
    else:
        s["A"] = psk.I8(s["codes"], s["scales"], cols=case["cols"])
        s["y"] = torch.empty((n, case["rows"]), dtype=TYPES[case["dtype"]], device="cuda")
        s["ws"] = psk.psk_linear_i8_workspace(s["A"], s["x"]) if op == "linear" else psk.psk_gemm_i8_workspace(s["A"], n)


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state, op)
    if op == "embed":
        return _embed_plain(state)
    if op == "grad":
        return _grad_plain(state)
    return _product_plain(state)


def _run_own(s, op):
    psk = s["psk"]
    if op == "embed":
        return psk.psk_embed(s["ids"], s["E"], s["y"], factor=s["factor"])
    if op == "grad":
        return psk.psk_embed_grad(s["ids"], s["dy"], s["de"], factor=s["factor"], ws=s["ws"])
    if op == "linear":
        return psk.psk_linear_i8(s["A"], s["x"], s["y"], bias=s["bias"], ws=s["ws"])
    return psk.psk_gemm_i8(s["A"], s["xcodes"], s["xscales"], s["y"], bias=s["bias"], ws=s["ws"])


def _embed_plain(s):
    case, ids = s["case"], s["ids"].long()
    at = ids.clamp(min=0)
    if case["table"] == "i8":
        rows = s["codes"][at][:, :case["dim"]].float() * s["scales"][at, None]
    else:
        rows = s["table"][at].float()
    return torch.where(ids[:, None] >= 0, rows * s["factor"], 0.0).to(TYPES[case["dtype"]])


def _grad_plain(s):
    case, ids = s["case"], s["ids"].long()
    de = torch.zeros((case["vocab"], case["dim"]), device="cuda")
    de.index_add_(0, ids.clamp(min=0), torch.where(ids[:, None] >= 0, s["dy"].float() * s["factor"], 0.0))
    return de.to(TYPES[case["gtype"]])


def _product_plain(s):
    case, cols = s["case"], s["case"]["cols"]
    if case["op"] == "linear":
        x = s["x"].double()
        top = x.abs().amax(1, keepdim=True)
        q = torch.where(top > 0, torch.round(127 * x / top), 0.0).float()
        xs = (top[:, 0] / 127).float()
    else:
        q, xs = s["xcodes"][:, :cols].float(), s["xscales"]
    y = (q @ s["codes"][:, :cols].float().t()) * s["scales"] * xs[:, None]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(TYPES[case["dtype"]])


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, n, es = case["op"], case["n"], BYTES[case["dtype"]]
    if op == "embed":
        # rows that are read: the expected number of different tokens
        tokens = n * (1 - case["holes"])
        distinct = float((1 - (1 - _chances(case["vocab"], "cpu")) ** tokens).sum())
        each = case["dim"] * BYTES[case["table"]] + (4 if case["table"] == "i8" else 0)
        return {"bytes": int(distinct * each) + n * (4 + case["dim"] * es), "flops": int(tokens * case["dim"])}
    if op == "grad":
        tokens = n * (1 - case["holes"])
        return {"bytes": 4 * n + int(tokens * case["dim"] * es) + case["vocab"] * case["dim"] * BYTES[case["gtype"]], "flops": int(2 * tokens * case["dim"])}
    rows, cols = case["rows"], case["cols"]
    return {"bytes": rows * (cols + 4 + (4 if case["bias"] else 0)) + n * (cols * es if op == "linear" else cols + 4) + n * rows * es,
            "flops": 2 * rows * cols * n}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        keep = (s["ids"] >= 0).nonzero()[:, 0]
        y = torch.zeros((case["n"], case["dim"]), dtype=torch.float64, device="cuda")
        which = s["ids"].index_select(0, keep)
        if case["table"] == "i8":
            y[keep] = s["codes"].index_select(0, which).double()[:, :case["dim"]] * (s["factor"] * s["scales"].double().index_select(0, which)).unsqueeze(1)
        else:
            y[keep] = s["factor"] * s["table"].index_select(0, which).double()
        return y
    if case["op"] == "grad":
        # tokens in ascending order, 8192 positions at a time
        de = torch.zeros((case["vocab"], case["dim"]), dtype=torch.float64, device="cuda")
        ids, order = torch.sort(s["ids"])
        first = int((ids < 0).sum())
        ids, order = ids[first:], order[first:]
        for r in range(0, ids.numel(), 8192):
            de.index_put_((ids[r:r + 8192].long(),), s["dy"][order[r:r + 8192]].double(), accumulate=True)
        return de * s["factor"]
    cols = case["cols"]
    if case["op"] == "linear":
        x = s["x"].double()
        top = x.abs().max(1)[0]
        xs = torch.where(top > 0, top / 127, 1.0)
        q = (x / xs[:, None]).round()
        # next to a border: 254 |x| on this or that side of (2k + 1) top, which 64 bits hold without rounding
        k = ((254 * x.abs()) / (2 * top.clamp(min=1e-300))[:, None]).floor()
        twice = 254 * x.abs() - (2 * k + 1) * top[:, None]
        up = (twice > 0) | ((twice == 0) & (k % 2 == 1))
        q = torch.where(top[:, None] > 0, torch.sign(x) * (k + up.double()), torch.zeros_like(q))
        xs = xs.float().double()
    else:
        q, xs = s["xcodes"][:, :cols].double(), s["xscales"].double()
    y = torch.empty((case["n"], case["rows"]), dtype=torch.float64, device="cuda")
    for r in range(0, case["rows"], 4096):
        w = s["codes"][r:r + 4096, :cols].double() * s["scales"][r:r + 4096].double().unsqueeze(1)
        y[:, r:r + 4096] = torch.matmul(w, q.t()).t() * xs.unsqueeze(1)
    return y if s["bias"] is None else y + s["bias"].double()
