"""Host-side checks of the packed cache's entry points: NULL handles and arguments are refused
before any device work (no GPU needed)."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def kv():
    from paper_2609_17983_gb300 import build
    build.build()
    from paper_2609_17983_gb300 import kvrepair
    return kvrepair


def test_null_handles_rejected(kv):
    lib = kv._lib
    out = ctypes.c_void_p(5)
    one = np.array([0], np.int32)
    p = one.ctypes.data
    assert lib.kvr_packed_create(None, 10, ctypes.byref(out)) == 1
    assert lib.kvr_packed_len(None) == -1
    assert lib.kvr_packed_write(None, p, 1, 0, 1, p, p) == 1
    assert lib.kvr_packed_read(None, p, 1, 0, 1, p, p) == 1
    assert lib.kvr_packed_bounds(None, 0, p, p, p) == 1
    assert lib.kvr_rows_create(None, p, p, 1, p, ctypes.byref(out)) == 1
    assert lib.kvr_rows_move(None, p) == 1
    assert lib.kvr_packed_attention(None, 0, p, 64, p) == 1
    assert lib.kvr_packed_select(None, 0, p, 64, 1, p) == 1
    assert lib.kvr_packed_attention_blocks(None, 0, p, 64, p, 1, p) == 1
    assert lib.kvr_pack(None, ctypes.byref(out)) == 1
    assert lib.kvr_packed_repair(None, p, 0, 1, p, 0) == 1
    assert lib.kvr_packed_logits(None, None, p, 1, 0, p) == 1
    assert b"NULL" in lib.kvr_last_error()
    lib.kvr_packed_free(None)
    lib.kvr_rows_free(None)


def test_every_packed_entry_point_is_bound(kv):
    for name in ("kvr_packed_create", "kvr_packed_write", "kvr_packed_read", "kvr_rows_create",
                 "kvr_packed_attention", "kvr_packed_select", "kvr_packed_attention_blocks",
                 "kvr_pack", "kvr_packed_repair", "kvr_packed_logits"):
        assert name in kv.EXPORTED and callable(getattr(kv, name))
    assert kv.BLOCK == 64
