"""The gradient of the embedding lookup in each of its ways: one launch, ranges of rows, digits counted by each workgroup, digits scanned."""
import numpy as np
import pytest

import ends_ref as R
from test_gpu_embed import TYPES, gradient, ints

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
