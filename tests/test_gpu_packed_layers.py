"""Layers of a packed document that were not written at a position: zeros, and bounds that know
of them."""
import numpy as np
import pytest
import torch

from paper_2609_17983_gb300 import synth
from tests import packed_plain as pp
from tests.test_gpu_packed import (SHAPES, TORCH, check, f64, kv, models, queries,  # noqa: F401
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


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,ask,blocks,grow", [(100, 8, 0, 1), (100, 8, 2, 28), (120, 40, 0, 30),
                                               (128, 64, 3, 64), (127, 2, 0, 2)])
def test_nothing_is_left_of_a_question(dtype, n, ask, blocks, grow):
    """The rows of a question leave the positions behind the document as they were: zeros where a
    write of one layer then lengthens it."""
    if kv is None:
        pytest.fail("no library")
    cfg = synth.preset("tiny", dtype=dtype)
    G, dh, L = cfg["n_kv_heads"], cfg["head_dim"], cfg["n_layers"]
    m = kv.Model(cfg, None, seed=0, max_context=512, max_rows=64)
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    cache = m.prefill(synth.document(1, n, cfg["vocab"]))
    doc = m.pack(cache)
    cache.close()
    before = read(doc, np.arange(n), L, G, dh, dtype)
    bounds = [doc.bounds(l) for l in range(L)]
    first = m.packed_logits(doc, synth.fill_tokens(5, ask, cfg["vocab"], cfg["delim_id"]), blocks)
    assert np.isfinite(first).all() and doc.n == n
    for l in range(L):
        assert all(same(a, b) for a, b in zip(doc.bounds(l), bounds[l]))
    new = rows(3, grow, 1, G, dh, dtype)
    doc.write(np.arange(n, n + grow), new, new, layer_begin=1, layer_end=2)
    x = pp.stored(f64(new))[:, 0]
    for l in range(L):
        tail = x if l == 1 else np.zeros_like(x)
        check_layer(doc, m, l, np.r_[before[0][:, l], tail], np.r_[before[1][:, l], tail], dtype,
                    cfg["n_heads"])
    doc.close()
    m.close()
