"""Operators of serving large language models that are measured: products with 4-bit weights, the router of a mixture of
experts, and its layer with 16-bit and with 4-bit weights.

Every case is one call with its sizes.  prepare() makes what a serving program holds: the weights as they are stored, the
activations of this step, output buffers and workspaces.  With `own` false run() computes the plain form with elementary torch
operations in 32 bits (the router's logits in 64: which expert is chosen turns on the last bits where two are close).
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # a small projection for one token: launch latency counts
        {"name": "q4_mv_small", "op": "q4", "rows": 1024, "cols": 1024, "n": 1, "dtype": "bf16", "group": 128, "zeros": False},
        # a square projection of a medium model, one token, with zero points
        {"name": "q4_mv", "op": "q4", "rows": 4096, "cols": 4096, "n": 1, "dtype": "f16", "group": 128, "zeros": True},
        # the output layer over a vocabulary, one token
        {"name": "q4_mv_large", "op": "q4", "rows": 32768, "cols": 8192, "n": 1, "dtype": "bf16", "group": 64, "zeros": False},
        # sixteen sequences decoded together
        {"name": "q4_mm_batch", "op": "q4", "rows": 10240, "cols": 4096, "n": 16, "dtype": "bf16", "group": 128, "zeros": True},
        # sizes that fill no tile, activations in 32 bits, three tokens, small groups
        {"name": "q4_mm_odd", "op": "q4", "rows": 5003, "cols": 2051, "n": 3, "dtype": "f32", "group": 32, "zeros": True},
        # a short prompt, or drafted tokens of several sequences
        {"name": "q4_mm_many", "op": "q4", "rows": 8192, "cols": 4096, "n": 64, "dtype": "f16", "group": 128, "zeros": False},
        # the router for one token
        {"name": "route_one", "op": "route", "n": 1, "dim": 2048, "experts": 64, "top_k": 6, "dtype": "bf16", "wtype": "bf16",
         "score": "softmax", "normalise": True, "bias": False},
        # the router for a batch, scores by a sigmoid with a balancing bias, router weights in 32 bits
        {"name": "route_batch", "op": "route", "n": 64, "dim": 4096, "experts": 160, "top_k": 8, "dtype": "bf16", "wtype": "f32",
         "score": "sigmoid", "normalise": True, "bias": True},
        # the layer for one token
        {"name": "moe_one", "op": "moe", "n": 1, "dim": 2048, "inter": 1024, "experts": 64, "top_k": 6, "dtype": "bf16", "empty": 0},
        # a batch of sequences: nearly every expert is read
        {"name": "moe_batch", "op": "moe", "n": 24, "dim": 4096, "inter": 1280, "experts": 32, "top_k": 4, "dtype": "f16", "empty": 0},
        # the layer in 4 bits for one token
        {"name": "moe_q4_one", "op": "moe_q4", "n": 1, "dim": 4096, "inter": 2048, "experts": 32, "top_k": 4, "dtype": "bf16",
         "empty": 0, "group": 128, "zeros": True},
        # a padded batch in 4 bits: five tokens go to no expert, an inner size that fills no tile
        {"name": "moe_q4_batch", "op": "moe_q4", "n": 48, "dim": 2048, "inter": 1000, "experts": 64, "top_k": 8, "dtype": "f16",
         "empty": 5, "group": 64, "zeros": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["q4", "q4", "route", "moe", "moe_q4"])
    half = rng.choice(["f16", "bf16"])
    if op == "q4":
        n = rng.choice([1, 1, rng.randint(2, 16), rng.randint(17, 64)])
        cols = _log(rng, 256, 16384)
        rows = _log(rng, 256, min(32768, 260_000_000 // cols // (1 if n <= 16 else 4)))
        if rng.random() < 0.5:
            rows, cols = (rows + 63) // 64 * 64, (cols + 127) // 128 * 128
        return {"op": op, "rows": rows, "cols": cols, "n": n, "dtype": rng.choice([half, half, "f32"]),
                "group": rng.choice([32, 64, 128, 128]), "zeros": rng.random() < 0.5}
    if op == "route":
        experts = rng.randint(8, 160)
        return {"op": op, "n": _log(rng, 1, 64), "dim": _log(rng, 256, 4096), "experts": experts, "top_k": rng.randint(1, 8),
                "dtype": rng.choice([half, half, "f32"]), "wtype": "f32", "score": rng.choice(["softmax", "sigmoid"]),
                "normalise": rng.random() < 0.5, "bias": rng.random() < 0.5}
    experts, n = rng.choice([8, 16, 32, 60, 64]), _log(rng, 1, 48)
    dim = _log(rng, 256, 4096)
    inter = _log(rng, 128, min(4096, 160_000_000 // experts // dim))
    if rng.random() < 0.5:
        dim, inter = (dim + 63) // 64 * 64, max(64, inter // 64 * 64)
    c = {"op": op, "n": n, "dim": dim, "inter": inter, "experts": experts, "top_k": rng.randint(1, 8), "dtype": half,
         "empty": rng.randint(0, n // 4)}
    return dict(c, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5) if op == "moe_q4" else c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + 29)
    return g


def _normal(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(TYPES[dtype])


def _activations(n, dim, dtype, g):
    """About normal, one feature in a hundred ten times as large (as the residual stream of a trained model has)."""
    x = torch.randn((n, dim), generator=g, device="cuda")
    big = torch.rand((1, dim), generator=g, device="cuda") < 0.01
    return torch.where(big, 10 * x, x).to(TYPES[dtype])


def _q4(count, rows, cols, group, zeros, stype, g):
    """(codes, scales, zeros) of `count` matrices; a row of codes takes a multiple of 16 bytes.  Weights of about 1/sqrt(cols)."""
    ldq, groups = (cols + 31) // 32 * 16, (cols + group - 1) // group
    codes = torch.randint(0, 256, (count, rows, ldq), generator=g, device="cuda", dtype=torch.uint8)
    s = (0.5 + torch.rand((count, rows, groups), generator=g, device="cuda")) / (4.6 * math.sqrt(cols))
    z = torch.randint(4, 13, (count, rows, groups), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return codes, s.to(TYPES[stype]), z


def _gating(n, experts, top_k, empty, g):
    """ids and gates of n tokens: distinct experts in a random order (a token cannot have more of them than there are), the
    last `empty` tokens have none."""
    k = min(top_k, experts)
    ids = torch.full((n, top_k), -1, dtype=torch.int32, device="cuda")
    ids[:, :k] = torch.rand((n, experts), generator=g, device="cuda").argsort(1)[:, :k].to(torch.int32)
    gates = torch.softmax(torch.randn((n, top_k), generator=g, device="cuda"), 1)
    if empty:
        ids[n - empty:] = -1
    gates[ids < 0] = 0
    return ids, gates


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = {"case": case}
    if op == "q4":
        s["x"] = _activations(case["n"], case["cols"], case["dtype"], g)
        stype = case["dtype"]
        s["w"] = tuple(None if t is None else t[0] for t in _q4(1, case["rows"], case["cols"], case["group"], case["zeros"], stype, g))
    elif op == "route":
        s["x"] = _activations(case["n"], case["dim"], case["dtype"], g)
        s["w"] = _normal((case["experts"], case["dim"]), case["wtype"], g, 1 / math.sqrt(case["dim"]))
        s["bias"] = torch.rand(case["experts"], generator=g, device="cuda") * 0.2 - 0.1 if case["bias"] else None
    else:
        n, dim, inter, experts = case["n"], case["dim"], case["inter"], case["experts"]
        s["x"] = _activations(n, dim, case["dtype"], g)
        s["ids"], s["gates"] = _gating(n, experts, case["top_k"], case["empty"], g)
        if op == "moe":
            s["w1"] = _normal((experts, inter, dim), case["dtype"], g, 1 / math.sqrt(dim))
            s["w3"] = _normal((experts, inter, dim), case["dtype"], g, 1 / math.sqrt(dim))
            s["w2"] = _normal((experts, dim, inter), case["dtype"], g, 1 / math.sqrt(inter))
        else:
            s["w1"] = _q4(experts, inter, dim, case["group"], case["zeros"], case["dtype"], g)
            s["w3"] = _q4(experts, inter, dim, case["group"], case["zeros"], case["dtype"], g)
            s["w2"] = _q4(experts, dim, inter, case["group"], case["zeros"], case["dtype"], g)
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program of the framework keeps beside the tensors: descriptions of 4-bit matrices, outputs, workspaces."""
    import paper_2001_00532_amd as psk

    case = s["case"]
    op, n = case["op"], case["n"]
    s["psk"] = psk
    if op == "q4":
        s["A"] = psk.Q4(*s["w"], cols=case["cols"], group=case["group"])
        s["y"] = torch.empty((n, case["rows"]), dtype=s["x"].dtype, device="cuda")
        s["ws"] = psk.psk_gemm_q4_workspace(s["A"], s["x"])
    elif op == "route":
        s["ids"] = torch.empty((n, case["top_k"]), dtype=torch.int32, device="cuda")
        s["gates"] = torch.empty((n, case["top_k"]), dtype=torch.float32, device="cuda")
        s["ws"] = psk.psk_moe_route_workspace(n, case["experts"])
    else:
        if op == "moe_q4":
            for w, cols in (("w1", case["dim"]), ("w3", case["dim"]), ("w2", case["inter"])):
                s["q" + w] = psk.Q4(*s[w], cols=cols, group=case["group"])
        s["y"] = torch.empty_like(s["x"])
        s["ws"] = psk.psk_moe_workspace(n, case["dim"], case["inter"], case["experts"], case["top_k"])


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state, op)
    if op == "q4":
        w = _dequantised(*state["w"], state["case"]["cols"], state["case"]["group"])
        return (state["x"].float() @ w.t()).to(state["x"].dtype)
    if op == "route":
        return _route_plain(state)
    return _moe_plain(state)


def _run_own(s, op):
    psk, case = s["psk"], s["case"]
    if op == "q4":
        return psk.psk_gemm_q4(s["A"], s["x"], s["y"], ws=s["ws"])
    if op == "route":
        score = psk.PSK_SCORE_SOFTMAX if case["score"] == "softmax" else psk.PSK_SCORE_SIGMOID
        return psk.psk_moe_route(s["x"], s["w"], s["ids"], s["gates"], score=score, bias=s["bias"], normalise=case["normalise"],
                                 factor=1.0, ws=s["ws"])
    if op == "moe":
        return psk.psk_moe_experts(s["x"], s["ids"], s["gates"], s["w1"], s["w3"], s["w2"], s["y"], act=psk.PSK_ACT_SILU, ws=s["ws"])
    return psk.psk_moe_experts_q4(s["x"], s["ids"], s["gates"], s["qw1"], s["qw3"], s["qw2"], s["y"], act=psk.PSK_ACT_SILU, ws=s["ws"])


def _dequantised(codes, scales, zeros, cols, group):
    """(q - z) * s of one matrix in 32 bits: the low half of a byte is the even column."""
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)[..., :cols].float()
    z = 8.0 if zeros is None else zeros.float().repeat_interleave(group, -1)[..., :cols]
    return (q - z) * scales.float().repeat_interleave(group, -1)[..., :cols]


def _route_plain(s):
    case = s["case"]
    logits = s["x"].double() @ s["w"].double().t()
    if case["score"] == "softmax":
        e = torch.exp(logits - logits.max(1, keepdim=True)[0])
        p = e / e.sum(1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-logits))
    key = logits if s["bias"] is None else p + s["bias"].double()
    order = torch.sort(key, dim=1, descending=True, stable=True)[1]
    k = min(case["top_k"], case["experts"])
    ids = torch.full((case["n"], case["top_k"]), -1, dtype=torch.int32, device="cuda")
    gates = torch.zeros((case["n"], case["top_k"]), dtype=torch.float64, device="cuda")
    ids[:, :k] = order[:, :k].to(torch.int32)
    gates[:, :k] = p.gather(1, order[:, :k])
    if case["normalise"]:
        gates = gates / gates.sum(1, keepdim=True)
    return ids, gates.float()


def _moe_plain(s):
    case = s["case"]
    x, ids, gates = s["x"].float(), s["ids"], s["gates"]
    y = torch.zeros_like(x)
    for e in range(case["experts"]):
        token, slot = (ids == e).nonzero(as_tuple=True)
        if token.numel() == 0:
            continue
        if case["op"] == "moe":
            w1, w3, w2 = s["w1"][e].float(), s["w3"][e].float(), s["w2"][e].float()
        else:
            w1, w3, w2 = (_dequantised(c[e], sc[e], None if z is None else z[e], cols, case["group"])
                          for (c, sc, z), cols in ((s["w1"], case["dim"]), (s["w3"], case["dim"]), (s["w2"], case["inter"])))
        a = x[token] @ w1.t()
        h = a / (1 + torch.exp(-a)) * (x[token] @ w3.t())
        y[token] += gates[token, slot, None] * (h @ w2.t())
    return y.to(s["x"].dtype)


# ------------------------------------------------------------------ what a pass cannot do without
def _q4_bytes(rows, cols, group, zeros, dtype):
    return rows * ((cols + 1) // 2) + rows * ((cols + group - 1) // group) * (BYTES[dtype] + (1 if zeros else 0))


def work(case):
    op, n, es = case["op"], case["n"], BYTES[case["dtype"]]
    if op == "q4":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": _q4_bytes(rows, cols, case["group"], case["zeros"], case["dtype"]) + n * (rows + cols) * es,
                "flops": 2 * rows * cols * n}
    if op == "route":
        return {"bytes": n * case["dim"] * es + case["experts"] * (case["dim"] * BYTES[case["wtype"]] + (4 if case["bias"] else 0)) +
                8 * n * case["top_k"], "flops": 2 * n * case["dim"] * case["experts"]}
    dim, inter, experts = case["dim"], case["inter"], case["experts"]
    k, tokens = min(case["top_k"], experts), n - case["empty"]
    # experts that are read: the expected number of those that some token goes to
    active = experts * (1 - (1 - k / experts) ** tokens)
    if op == "moe":
        each = 3 * dim * inter * es
    else:
        each = 2 * _q4_bytes(inter, dim, case["group"], case["zeros"], case["dtype"]) + \
            _q4_bytes(dim, inter, case["group"], case["zeros"], case["dtype"])
    return {"bytes": int(active * each) + 2 * n * dim * es + 8 * n * case["top_k"], "flops": 6 * tokens * k * dim * inter}


# ------------------------------------------------------------------ the definition in 64 bits
def _weights64(codes, scales, zeros, cols, group):
    j = torch.arange(cols, device=codes.device)
    q = (codes[:, j // 2].to(torch.int32) >> (4 * (j % 2)).to(torch.int32)) & 15
    at = j // group
    z = 8 if zeros is None else zeros[:, at].to(torch.int32)
    return (q - z).double() * scales.double()[:, at]


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"] == "q4":
        codes, scales, zeros = s["w"]
        y = torch.empty((case["n"], case["rows"]), dtype=torch.float64, device=x.device)
        for r in range(0, case["rows"], 4096):
            part = slice(r, r + 4096)
            y[:, part] = torch.matmul(_weights64(codes[part], scales[part], None if zeros is None else zeros[part], case["cols"],
                                                 case["group"]), x.t()).t()
        return y
    if case["op"] == "route":
        l = (x[:, None, :] * s["w"].double()[None]).sum(2) if case["n"] <= 8 else torch.matmul(s["w"].double(), x.t()).t()
        p = torch.softmax(l, 1) if case["score"] == "softmax" else torch.sigmoid(l)
        key = (l if s["bias"] is None else p + s["bias"].double()).cpu().tolist()
        ids = torch.full((case["n"], case["top_k"]), -1, dtype=torch.int32)
        for t, row in enumerate(key):
            best = sorted(range(len(row)), key=lambda e: (-row[e], e))[:case["top_k"]]
            ids[t, :len(best)] = torch.tensor(best, dtype=torch.int32)
        ids = ids.to(x.device)
        gates = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0).long()), 0.0)
        return ids, gates / gates.sum(1, keepdim=True) if case["normalise"] else gates
    y = torch.zeros_like(x)
    for e in sorted(set(s["ids"].flatten().tolist()) - {-1}):
        if case["op"] == "moe":
            w1, w3, w2 = s["w1"][e].double(), s["w3"][e].double(), s["w2"][e].double()
        else:
            def of(w, cols):
                return _weights64(w[0][e], w[1][e], None if w[2] is None else w[2][e], cols, case["group"])
            w1, w3, w2 = of(s["w1"], case["dim"]), of(s["w3"], case["dim"]), of(s["w2"], case["inter"])
        weight = torch.where(s["ids"] == e, s["gates"].double(), 0.0).sum(1)
        who = (s["ids"] == e).any(1).nonzero()[:, 0]
        a = torch.matmul(w1, x[who].t())
        h = a * torch.sigmoid(a) * torch.matmul(w3, x[who].t())
        y.index_add_(0, who, torch.matmul(w2, h).t() * weight[who, None])
    return y
