"""Documents held in 4 bits: prefilled, packed, edited, repaired in place, and asked a question.

One document of each size is prefilled and packed (its bf16 cache is dropped), an edit is repaired
in the packed entries (the span and the positions after it), and a query is answered over all
positions and over the blocks that its bounds select.  Prints the bytes of either cache, the times,
and how far the packed answers lie from those of the repaired bf16 cache (the weights are random:
their attention is nearly flat, so the answers hang on small differences of large means, and a
query that reads a fifth of the blocks answers another question).

    python examples/packed_documents.py [--preset llama8b] [--layers 4] [--n 5000] [--blocks 32]
"""
import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_17983_gb300 import kvrepair as kv  # noqa: E402
from paper_2609_17983_gb300 import synth  # noqa: E402


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--preset", default="llama8b", choices=sorted(synth.PRESETS))
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--n", type=int, default=5000)
    ap.add_argument("--blocks", type=int, default=32)
    a = ap.parse_args()
    cfg = synth.preset(a.preset, n_layers=a.layers)
    model = kv.Model(cfg, None, seed=0, max_context=16384, max_rows=4096)
    rows = a.n * a.layers * cfg["n_kv_heads"] * cfg["head_dim"] * 2
    print(f"{a.preset}, {a.layers} layers, {a.n} positions: "
          f"{rows * (2 if cfg['dtype'] == 'bf16' else 4) / 1e6:.1f} MB of K/V, "
          f"{rows * 9 / 16 / 1e6:.1f} MB packed")

    doc = synth.document(1, a.n, cfg["vocab"])
    span = a.n // 2
    new = synth.fill_tokens(7, 8, cfg["vocab"], cfg["delim_id"])
    after = np.arange(span + 8, min(a.n, span + 40))
    query = synth.fill_tokens(5, 8, cfg["vocab"], cfg["delim_id"])

    def timed(what, f):
        f()
        model.synchronize()
        t = time.perf_counter()
        out = f()
        model.synchronize()
        print(f"  {what}: {(time.perf_counter() - t) * 1e3:.3f} ms")
        return out

    cache = model.prefill(doc)
    packed = timed("pack", lambda: model.pack(cache))
    timed("repair in bf16", lambda: cache.repair(new, span, after))
    timed("repair in 4 bits", lambda: packed.repair(new, span, after))
    ref = timed("query over the cache", lambda: model.logits(cache, query))
    full = timed("query over the packed document", lambda: model.packed_logits(packed, query))
    some = timed(f"query over {a.blocks} blocks of it",
                 lambda: model.packed_logits(packed, query, a.blocks))
    for name, x in (("packed", full), ("packed, selected blocks", some)):
        print(f"  {name}: logits differ by {np.abs(x - ref).max() / np.abs(ref).max():.3f} of the "
              f"largest, correlation {np.corrcoef(x, ref)[0, 1]:.4f}")
    packed.close()
    cache.close()
    model.close()


if __name__ == "__main__":
    main()
