"""Queries with an infinite entry over packed documents: NaN where the row sees a key."""
import numpy as np
import pytest
import torch

from tests import packed_plain as pp
from tests.test_gpu_packed import SHAPES, check, f64, models, queries, rows  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype,n,R", [
    ("dh128", "bf16", 300, 4), ("dh64", "fp32", 300, 4), ("dh128", "fp32", 5000, 4),
    ("dh128", "bf16", 12345, 36), ("dh64", "bf16", 4000, 1201)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_query(models, shape, dtype, n, R, sign):  # noqa: F811
    """Where all of a channel's keys have one sign, an infinite entry of the query makes all scores
    -infinity (or all +infinity): their softmax is NaN, not the zeros of a row without keys."""
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    k, v = rows(n, n, 2, G, dh, dtype), rows(n + 1, n, 2, G, dh, dtype)
    k[..., 5] = -8 - k[..., 5].abs()
    doc = m.packed(n)
    doc.write(np.arange(n), k, v)
    pos = np.arange(n - R, n)
    pos[0] = -1
    r = m.rows([(doc, pos)])
    q = queries(R, R, H, dh, dtype)
    for row, head in ((0, 0), (1, H - 1), (R // 2, 1), (R - 1, 0)):
        q[row, head, 5] = sign * float("inf")
    out = torch.empty_like(q)
    r.attention(1, q, out)
    some = np.unique([0, 1, 2, R // 2, R - 2, R - 1])
    with np.errstate(invalid="ignore"):
        check(f64(out)[some], f64(q)[some], pos[some], pp.stored(f64(k))[:, 1],
              pp.stored(f64(v))[:, 1], dtype)
    assert np.isnan(f64(out)).any(2).sum() == 3  # the first row sees nothing
    r.close()
    doc.close()
