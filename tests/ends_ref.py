"""Plain 64-bit forms of the products of 8-bit integers, of the embedding and of its gradient, with the bounds of their errors.

A product or sum of 32 bits is off by at most 2^-24 of its result; a sum of k terms, in any order, by k 2^-24 times the sum of the terms' sizes.
"""
import numpy as np
import torch

from serving_ref import check, out_error  # noqa: F401

ULP = 2.0 ** -24


def quantised(x):
    """(codes int64, scales float32) of the rows of x, from whole numbers: 254 |x| against (2k + 1) m is exact in 64 bits."""
    a = x.double().numpy()
    m = np.abs(a).max(1, initial=0.0) if a.shape[1] else np.zeros(a.shape[0])
    bad = ~np.isfinite(m)
    ok = (m > 0) & ~bad
    safe = np.where(ok, m, 1.0)[:, None]
    finite = np.where(bad[:, None], 0.0, np.nan_to_num(a))
    k = np.floor(127 * np.abs(finite) / safe)
    k = np.where(254 * np.abs(finite) < 2 * k * safe, k - 1, k)                  # the quotient was rounded up to a whole number
    d = 254 * np.abs(finite) - (2 * k + 1) * safe
    c = k + ((d > 0) | ((d == 0) & (k % 2 == 1)))
    codes = np.where(ok[:, None], np.sign(finite) * c, 0.0)
    scales = np.where(bad, np.float32("nan"), np.where(bad, 0, m).astype(np.float32) / np.float32(127))
    return torch.from_numpy(codes).to(torch.int64), torch.from_numpy(scales.astype(np.float32))


def product(q, a, sa, sq, bias, dtype):
    """(y, bound) for codes q of tokens (n x cols) and a of channels (rows x cols), int64."""
    s = (q.double() @ a.double().t()) * sa.double() * sq.double()[:, None]      # sums below 2^31 are exact in 64 bits
    y = s if bias is None else s + bias.double()
    # from half a step above the largest number on, rounding to nearest gives infinity (f16: 65504 + 16)
    y = torch.where(y.abs() >= torch.finfo(dtype).max * (1 + torch.finfo(dtype).eps / 4), torch.sign(y) * float("inf"), y)
    return y, 3 * ULP * s.abs() + ULP * y.abs() + out_error(y, dtype)


def embed(ids, table, factor, dtype, scales=None):
    """(y, bound)."""
    rows = table.shape[0]
    y = torch.zeros(ids.numel(), table.shape[1], dtype=torch.float64)
    for t, v in enumerate(ids.tolist()):
        if 0 <= v < rows:
            y[t] = table[v].double() * factor * (1.0 if scales is None else float(scales[v]))
    return y, 2 * ULP * y.abs() + out_error(y, dtype)


def embed_grad(ids, dy, rows, factor, padding, dtype, old=None):
    """(dE, bound)."""
    de, size = (torch.zeros(rows, dy.shape[1], dtype=torch.float64) for _ in range(2))
    count = torch.zeros(rows, 1, dtype=torch.float64)
    for t, v in enumerate(ids.tolist()):
        if 0 <= v < rows and v != padding:
            de[v] += dy[t].double()
            size[v] += dy[t].double().abs()
            count[v] += 1
    y = de * factor if old is None else old.double() + de * factor
    bound = (count + 2) * ULP * size * abs(factor) + 2 * ULP * y.abs() + out_error(y, dtype)
    if old is not None:                                     # a row that no token has is not touched
        bound = torch.where(count > 0, bound, torch.full_like(bound, 1e-300))
    return y, bound
