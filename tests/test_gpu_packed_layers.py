"""Layers of a packed document that were not written at a position: zeros, and bounds that know
of them."""
import numpy as np
import pytest
import torch

from tests import packed_plain as pp
from tests.test_gpu_packed import (SHAPES, check, f64, models, queries,  # noqa: F401
                                   read, rows, same)

pytestmark = pytest.mark.gpu


def check_layer(doc, m, layer, k, v, dtype, H):
    """Rows, bounds, a choice of blocks and attention of one layer against k, v [n, G, dh]."""
    n, G, dh = k.shape
    got = read(doc, np.arange(n), 1, G, dh, dtype, layer_begin=layer, layer_end=layer + 1)
    assert same(got[0][:, 0], k) and same(got[1][:, 0], v)
    for a, b in zip(doc.bounds(layer), pp.bounds(k)):
        assert same(a, b)
    pos = np.array([n // 2, n - 1])
    r = m.rows([(doc, pos)])
    q = queries(n, 2, H, dh, dtype)
    out, blocks = torch.empty_like(q), torch.empty((2, G, 2), dtype=torch.int32, device="cuda")
    r.select(layer, q, blocks)
    assert np.array_equal(blocks.cpu().numpy(), pp.select(f64(q), pos, k, 2))
    r.attention(layer, q, out)
    check(f64(out), f64(q), pos, k, v, dtype)
    r.close()


@pytest.mark.parametrize("shape,dtype", [("dh64", "fp32"), ("dh128", "bf16")])
@pytest.mark.parametrize("steps", [
    [(0, 10), (1, 64)],            # within a block
    [(0, 10), (1, 300)],           # past it: blocks of zeros alone
    [(1, 128), (0, 129)],          # a block of one row
    [(0, 200), (1, 64), (1, 205), (0, 203)],  # and behind rows of the other layer
])
def test_layers_of_unequal_length(models, shape, dtype, steps):  # noqa: F811
    """Each step writes a layer from where it ends up to a length; keys all of one sign."""
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    n = max(s[1] for s in steps)
    doc = m.packed(n + 70)
    k, v = np.zeros((2, n, G, dh)), np.zeros((2, n, G, dh))
    at = [0, 0]
    for i, (layer, end) in enumerate(steps):
        where = np.arange(at[layer], end)
        a, b = rows(i, len(where), 1, G, dh, dtype).abs(), rows(i + 9, len(where), 1, G, dh, dtype)
        a[..., ::3] *= -1
        doc.write(where, a, b, layer_begin=layer, layer_end=layer + 1)
        k[layer, where], v[layer, where] = pp.stored(f64(a))[:, 0], pp.stored(f64(b))[:, 0]
        at[layer] = end
        for l in range(2):
            check_layer(doc, m, l, k[l, :doc.n], v[l, :doc.n], dtype, H)
    doc.close()
