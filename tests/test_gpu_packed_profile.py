"""The profile of passes over packed documents."""
import numpy as np
import pytest

from paper_2609_17983_gb300 import synth

try:
    from paper_2609_17983_gb300 import kvrepair as kv
except ImportError as _e:  # pragma: no cover
    kv, _IMPORT_ERROR = None, _e

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [20, 1200])
def test_a_layers_attention_is_counted_once(K):
    """Few rows and many, which go by way of unpacked pages: one attention a layer but the last."""
    if kv is None:
        raise _IMPORT_ERROR
    cfg = synth.preset("tiny", dtype="bf16", n_layers=3)
    n = 2000
    m = kv.Model(cfg, None, seed=0, max_context=2048, max_rows=2048)
    cache = m.prefill(synth.document(1, n, cfg["vocab"]))
    doc = m.pack(cache)
    cache.close()
    kv.kvr_profile_enable(m.h, True)
    kv.kvr_profile_reset(m.h)
    doc.repair([1], n - K - 1, np.arange(n - K, n))
    m.synchronize()
    got = kv.kvr_profile_read(m.h)
    kv.kvr_profile_enable(m.h, False)
    assert got["attention"]["launches"] == cfg["n_layers"] - 1
    doc.close()
    m.close()
