"""Attention and block selection over long packed documents, whose parts' sums meet through memory,
against the same in 64 bits on the stored values."""
import math

import numpy as np
import pytest
import torch

from paper_2609_17983_gb300 import synth
from tests.test_gpu_packed import TORCH, kv, queries

pytestmark = pytest.mark.gpu

# head size, heads, KV heads; with one KV head a long document has the most parts to add
SHAPES = {"dh64": (64, 4, 2), "dh128": (128, 14, 2), "dh128_9": (128, 18, 2), "dh64_1": (64, 3, 3),
          "dh128_one": (128, 7, 1), "dh64_one": (64, 4, 1)}


def model(shape, dtype):
    if kv is None:
        pytest.fail("no library")
    dh, H, G = SHAPES[shape]
    cfg = synth.preset("tiny", dtype=dtype, head_dim=dh, n_heads=H, n_kv_heads=G, n_layers=1)
    m = kv.Model(cfg, None, seed=0, max_context=256, max_rows=64)
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    return m


def long_document(m, seed, n, shape, dtype):
    """A document written in pieces, and its stored K and V [n, G, dh]."""
    dh, H, G = SHAPES[shape]
    g = torch.Generator(device="cuda").manual_seed(seed)
    doc = m.packed(n)
    channel = torch.exp(0.5 * torch.randn((G, dh), generator=g, device="cuda"))
    stored = [torch.empty((n, G, dh), dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    for p in range(0, n, 1 << 16):
        c = min(1 << 16, n - p)
        k, v = (torch.randn((c, 1, G, dh), generator=g, device="cuda") for _ in range(2))
        k = k * channel
        where = np.arange(p, p + c)
        doc.write(where, k.to(TORCH[dtype]), v.to(TORCH[dtype]))
        ko, vo = (x[p:p + c].unsqueeze(1) for x in stored)
        doc.read(where, ko, vo)
    return doc, stored[0], stored[1]


def reference(q, pos, k, v):
    """out, largest value and largest sum |q k| / sqrt(dh) [R, H, ...] in 64 bits."""
    R, H, dh = q.shape
    G = k.shape[1]
    out = torch.zeros((R, H, dh), dtype=torch.float64, device="cuda")
    vmax, smax = (torch.zeros((R, H, 1), dtype=torch.float64, device="cuda") for _ in range(2))
    for g in range(G):
        K, V = k[:, g].double(), v[:, g].double()
        for r in range(R):
            n = int(pos[r]) + 1
            if n == 0:
                continue
            heads = slice(g * (H // G), (g + 1) * (H // G))
            x = q[r, heads].double() @ K[:n].T / math.sqrt(dh)
            out[r, heads] = torch.softmax(x, 1) @ V[:n]
            vmax[r, heads] = V[:n].abs().max()
            smax[r, heads] = ((q[r, heads].double().abs() @ K[:n].abs().T).amax(1, True) /
                              math.sqrt(dh))
    return out, vmax, smax


def allowed(dtype, ref, vmax, smax, keys):
    """As for short documents, and the sums' additions: at most keys / 64 on the way of a key
    (they are dealt to all of the chip) and 1024 parts'."""
    delta = 2.0 ** -19 + 16 * 2.0 ** -23 * smax + (keys / 64 + 1024) * 2.0 ** -23
    if dtype == "bf16":
        return 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2 * delta) * vmax
    return 2 * delta * vmax + 2.0 ** -24 * ref.abs()


@pytest.mark.parametrize("shape,dtype,docs", [
    ("dh128", "bf16", [(131072, [131071])]),
    ("dh128", "fp32", [(131072, [131071])]),
    ("dh64", "bf16", [(40001, [-1, 17, 39999, 40000])]),
    ("dh64_1", "fp32", [(65537, [5, 65536])]),
    ("dh128_9", "bf16", [(20003, [20002]), (70, [69]), (1, [0]), (60000, [59998, 59999])]),
    ("dh64", "fp32", [(30000, [29000, 29999]), (100, [-1, 99]), (64000, [63999])]),
    ("dh128", "bf16", [(1 << 20, [(1 << 20) - 1])]),
    ("dh64", "fp32", [((1 << 20) - 3, [600000, (1 << 20) - 4])]),
    ("dh128_one", "bf16", [(1 << 20, [(1 << 20) - 1])]),
    ("dh64_one", "fp32", [((1 << 20) - 1, [(1 << 20) - 2])]),
])
def test_attention_of_long_documents(shape, dtype, docs):
    dh, H, G = SHAPES[shape]
    m = model(shape, dtype)
    made = [long_document(m, 7 * i + n, n, shape, dtype) for i, (n, _) in enumerate(docs)]
    r = m.rows([(d[0], np.array(p)) for d, (_, p) in zip(made, docs)])
    q = queries(r.n, r.n, H, dh, dtype)
    out = torch.full_like(q, float("nan"))
    r.attention(0, q, out)
    again = torch.full_like(q, float("nan"))
    r.attention(0, q, again)  # the arrivals' counters are zero again, and no sum's order changes
    assert torch.equal(out, again)
    i = 0
    for (doc, k, v), (n, pos) in zip(made, docs):
        x = slice(i, i + len(pos))
        ref, vmax, smax = reference(q[x], pos, k, v)
        err = (out[x].double() - ref).abs() - allowed(dtype, ref, vmax, smax, n)
        assert not bool((err > 0).any()), float(err.max())
        assert bool(torch.isfinite(out[x]).all())
        i += len(pos)
    m.close()  # and its documents


@pytest.mark.parametrize("n,count", [(131072, 32), ((1 << 20) - 5, 100), (1 << 20, 9000)])
def test_selection_of_long_documents(n, count):
    """Scores from the document's own bounds: whole numbers and powers of two, so 64 bits are exact."""
    dh, H, G = SHAPES["dh128"]
    m = model("dh128", "bf16")
    doc, _, _ = long_document(m, n, n, "dh128", "bf16")
    pos = [n // 2, n - 1]
    r = m.rows([(doc, pos)])
    q = queries(n % 97, 2, H, dh, "bf16")
    blocks = torch.empty((2, G, count), dtype=torch.int32, device="cuda")
    r.select(0, q, blocks)
    hi, lo, unit = (x.astype(np.float64) for x in doc.bounds(0))
    x = q.float().cpu().numpy().reshape(2, G, H // G, dh)
    for row in range(2):
        own = pos[row] // 64
        for g in range(G):
            up, down = np.zeros(dh, np.float32), np.zeros(dh, np.float32)
            for h in range(H // G):  # in order, in 32 bits: part of the definition
                up += np.maximum(x[row, g, h], 0)
                down += np.minimum(x[row, g, h], 0)
            a = max(up.max(), -down.min())
            t = 2.0 ** math.ceil(math.log2(float(a) / 127))
            score = unit[g] * (hi[g] @ np.rint(up / t) + lo[g] @ np.rint(down / t))
            best = np.argsort(-score[:own], kind="stable")[:count - 1]
            want = np.full(count, -1)
            took = np.sort(np.r_[best, own])
            want[:len(took)] = took
            assert np.array_equal(blocks[row, g].cpu().numpy(), want)
    m.close()
