"""Attention over packed documents where one key takes nearly all of the weight: what the small
weights add up to, against the same in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_packed import SHAPES, TORCH, f64, models  # noqa: F401 (a fixture)
from tests import packed_plain as pp

pytestmark = pytest.mark.gpu


def allowed(dtype, ref, w, count, total, mean, gap):
    """What the roundings allow of a row's tail of `count` keys of weight w (the first key's is one,
    its value zero), values of mean `mean`, all weights `total`.

    A weight is rounded to 11 bits, the smallest to steps of half's subnormals, 2^-24, where the
    largest weight is 2^6 at least: off by w 2^-11 or 2^-31.  fp32: in two halves, 22 bits or,
    with the second 2^11 above the first and the largest weight 2^7 at least, 2^-43.  It moves
    the numerator and may move the sum.
    A score is off by 16 roundings of itself, an exponential by 2^-19, of the numerator and of
    the sum.  The sums are of 32 bits: fewer than count / 8 + 64 additions on the way of a
    key.  The output is rounded to its type."""
    step = np.maximum(w * 2.0 ** -11, 2.0 ** -31) if dtype == "bf16" else np.maximum(
        w * 2.0 ** -22, 2.0 ** -43)
    delta = 2 * (2.0 ** -19 + 16 * 2.0 ** -23 * gap) + (count / 8 + 64) * 2.0 ** -23
    return (step * count * (mean + np.abs(ref)) / total + delta * np.abs(ref) +
            2.0 ** (-8 if dtype == "bf16" else -24) * np.abs(ref))


@pytest.mark.parametrize("shape,dtype,n,R,many", [
    ("dh128", "bf16", 4096, 1, False), ("dh64", "bf16", 1500, 9, False),
    ("dh128", "fp32", 4096, 1, False), ("dh64", "fp32", 1500, 9, False),
    ("dh128", "fp32", 20000, 3, False),
    ("dh128", "bf16", 12345, 36, True), ("dh128", "bf16", 12345, 300, True),
    ("dh64", "bf16", 8000, 1201, True)])
def test_a_dominating_key(models, shape, dtype, n, R, many):  # noqa: F811
    """The first key's score is 8 to 20 nats above all others', its value is zero: the output is
    the others' alone, which are alike, so that a rounding of their weight does not average out."""
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    k = torch.zeros((n, 2, G, dh), dtype=TORCH[dtype], device="cuda")
    k[0, :, :, 0] = 6.0  # stored as it is
    g = torch.Generator(device="cuda").manual_seed(n + R)
    v = (torch.randn((n, 2, G, dh), generator=g, device="cuda").abs() + 0.5).to(TORCH[dtype])
    v[0] = 0
    doc = m.packed(n)
    doc.write(np.arange(n), k, v)
    q = torch.zeros((R, H, dh), dtype=TORCH[dtype], device="cuda")
    want = torch.linspace(8, 20, R * H, device="cuda").view(H, R).T  # every row and head its own
    q[:, :, 0] = (want * math.sqrt(dh) / 6).to(TORCH[dtype])
    pos = np.arange(n - R, n)
    r = m.rows([(doc, pos)])
    out = torch.full_like(q, float("nan"))
    before = m.launches()
    r.attention(1, q, out)
    assert m.launches() - before == 1 if not many else m.launches() - before >= 2
    tail = np.cumsum(pp.stored(f64(v[:, 1])), 0)[pos]  # [R, G, dh]
    gap = f64(q)[:, :, 0] * 6 / math.sqrt(dh)
    w = np.exp(-gap)
    total = 1 + w * pos[:, None]
    sums = tail.repeat(H // G, 1)
    ref = (w / total)[..., None] * sums
    x = [a[..., None] for a in (w, total, gap)]
    err = np.abs(f64(out) - ref) - allowed(dtype, ref, x[0], pos[:, None, None], x[1],
                                           sums / pos[:, None, None], x[2])
    assert not (err > 0).any(), float((err / ref).max())
    assert np.isfinite(f64(out)).all()
    r.close()
    doc.close()
