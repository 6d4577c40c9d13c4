"""Plain 64-bit forms of the products with 4-bit weights and of the mixture of experts, with the bounds of their errors.

Bounds.  A sum of k terms in 32 bits, in any order, is off by at most k 2^-23 times the sum of the terms' sizes (2^-23: the matrix
cores may cut off where other instructions round); rounding to a type by half a step, finfo(type).eps / 2 of the value.
"""
import math

import numpy as np
import torch

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
STEP = 2.0 ** -23


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def out_error(ref, dtype):
    """Rounding of the result, and the smallest number of the type."""
    return half_step(dtype) * ref.abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def q4_weights(rng, rows, cols, group, zeros, stype, count=None, pad=0, scale=0.05):
    """(codes, scales, zeros) on the CPU; rows of codes take `pad` * 16 bytes more than they need, all bytes random."""
    lead = (rows,) if count is None else (count, rows)
    ldq, groups = (cols + 31) // 32 * 16 + 16 * pad, (cols + group - 1) // group
    codes = torch.from_numpy(rng.integers(0, 256, lead + (ldq,), dtype=np.uint8))
    scales = torch.from_numpy(rng.uniform(0.2, 1.0, lead + (groups,)) * scale).to(stype)
    z = torch.from_numpy(rng.integers(0, 16, lead + (groups,), dtype=np.uint8)) if zeros else None
    return codes, scales, z


def dequantised(codes, scales, zeros, cols, group):
    """float64 rows x cols."""
    out = torch.zeros(codes.shape[0], cols, dtype=torch.float64)
    for j in range(cols):
        q = (codes[:, j // 2] >> 4) if j % 2 else (codes[:, j // 2] & 15)
        z = 8.0 if zeros is None else zeros[:, j // group].double()
        out[:, j] = (q.double() - z) * scales[:, j // group].double()
    return out


def gemm(w, x, dtype):
    """(y, bound) of x w^T for float64 weights."""
    x = x.double()
    y = x @ w.t()
    return y, (w.shape[1] + 64) * STEP * (x.abs() @ w.abs().t()) + out_error(y, dtype)


def act(v, kind):
    return v / (1 + torch.exp(-v)) if kind == 0 else 0.5 * v * (1 + torch.erf(v / math.sqrt(2)))


def layer(x, crd, vals, w1, w3, w2, kind, dtype, parts):
    """(y, bound): w1, w3, w2 lists of float64 matrices.  parts: relative error of a value between the two products, held as two
    16-bit numbers (half a step of the one times half a step of the other)."""
    x = x.double()
    n, dim = x.shape
    y, err = torch.zeros(n, dim, dtype=torch.float64), torch.zeros(n, dim, dtype=torch.float64)
    inter = w1[0].shape[0]
    for t in range(n):
        for s in range(crd.shape[1]):
            e, g = int(crd[t, s]), float(vals[t, s])
            if not 0 <= e < len(w1):
                continue
            a, u = w1[e] @ x[t], w3[e] @ x[t]
            ea, eu = (k * (w.abs() @ x[t].abs()) for k, w in (((dim + 64) * STEP, w1[e]), ((dim + 64) * STEP, w3[e])))
            h = act(a, kind) * u
            # |act'| <= 1.13; exp, erf, a division and two products: 16 steps of 32 bits; f16 parts: 2^-28 absolute
            eh = 1.13 * ea * (u.abs() + eu) + act(a, kind).abs() * eu + (16 * STEP + parts) * h.abs() + 2.0 ** -28
            y[t] += g * (w2[e] @ h)
            err[t] += abs(g) * (w2[e].abs() @ (eh + (inter + 64 + crd.shape[1]) * STEP * h.abs()))
    return y, err + out_error(y, dtype)


def route(x, w, top_k, score, bias, normalise, factor):
    """(ids, gates) per token.  Every logit is summed in the same order, so equal rows of w have equal ones (a library's product adds up
    the last columns of its result in another order than the first)."""
    l = torch.stack([torch.tensor([math.fsum((a * b).tolist()) for b in w.double()], dtype=torch.float64) for a in x.double()])
    p = torch.softmax(l, 1) if score == 0 else 1 / (1 + torch.exp(-l))
    key = l if bias is None else p + bias.double()
    ids = torch.full((x.shape[0], top_k), -1, dtype=torch.int32)
    gates = torch.zeros((x.shape[0], top_k), dtype=torch.float64)
    for t in range(x.shape[0]):
        allowed = [e for e in range(w.shape[0]) if bias is None or float(bias[e]) != -math.inf]

        def order(e):
            v = float(key[t, e])
            return (1, 0.0, e) if math.isnan(v) else (0, -v, e)
        chosen = sorted(allowed, key=order)[:top_k]
        total = sum(float(p[t, e]) for e in chosen)
        for s, e in enumerate(chosen):
            ids[t, s] = e
            gates[t, s] = float(p[t, e]) / (total if normalise else 1.0) * factor
    return ids, gates


def check(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, what
    special = ~torch.isfinite(ref)
    same = torch.isnan(got) == torch.isnan(ref)
    assert bool(same.all()), "%s: NaN at other places" % what
    inf = torch.isinf(ref)
    assert bool((got[inf] == ref[inf]).all()), "%s: infinities" % what
    off = ((got - ref).abs() / bound)[~special]
    worst = float(off.max()) if off.numel() else 0.0
    print("%s: worst error / bound %.3g" % (what, worst), flush=True)
    assert worst <= 1.0, "%s: worst error / bound %.3g" % (what, worst)
