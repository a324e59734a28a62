"""Packed documents through the model: packed from a cache, repaired in place, asked a question,
against a plain decoder in 64 bits (numpy, with the stored form's roundings)."""
import numpy as np
import pytest

from paper_2609_17983_gb300 import synth
from tests import packed_plain as pp

try:
    from paper_2609_17983_gb300 import kvrepair as kv
except ImportError as _e:  # pragma: no cover
    kv, _IMPORT_ERROR = None, _e

pytestmark = pytest.mark.gpu


def values(a, dtype):
    return (synth.bf16_bits_to_f32(a) if dtype == "bf16" else a).astype(np.float64)


def bf16(x):
    return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(x.astype(np.float32))).astype(np.float64)


class Plain:
    """Layers' stored K/V [L][cap, G, dh] and a pass of rows over them."""

    def __init__(self, cfg, W, k, v, cap):
        self.cfg, self.W = cfg, W
        self.round = bf16 if cfg["dtype"] == "bf16" else (lambda x: x)
        n, L, G, dh = k.shape
        self.k, self.v = np.zeros((L, cap, G, dh)), np.zeros((L, cap, G, dh))
        self.k[:, :n], self.v[:, :n] = k.transpose(1, 0, 2, 3), v.transpose(1, 0, 2, 3)

    def norm(self, h, g):
        return self.round(h / np.sqrt((h * h).mean(1, keepdims=True) + self.cfg["rms_eps"]) * g)

    def rope(self, x, pos):
        half = x.shape[2] // 2
        ang = pos[:, None] * self.cfg["rope_theta"] ** (-np.arange(half) * 2.0 / x.shape[2])
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        a, b = x[..., :half], x[..., half:]
        return np.concatenate([a * c - b * s, b * c + a * s], -1)

    def run(self, tokens, pos, n_blocks=0):
        """Rows `tokens` at positions pos (ascending); the last row's logits."""
        c, dt = self.cfg, self.cfg["dtype"]
        H, G, dh, M = c["n_heads"], c["n_kv_heads"], c["head_dim"], len(pos)
        h = values(self.W["embed"], dt)[tokens]
        for l in range(c["n_layers"]):
            w = {k: values(x, dt) for k, x in self.W["layers"][l].items() if x is not None}
            a = self.norm(h, w["attn_norm"])
            q = self.round(self.rope((a @ w["wq"].T).reshape(M, H, dh), pos))
            k = self.rope((a @ w["wk"].T).reshape(M, G, dh), pos)
            v = (a @ w["wv"].T).reshape(M, G, dh)
            self.k[l][pos], self.v[l][pos] = pp.stored(self.round(k)), pp.stored(self.round(v))
            end = pos[-1] + 1
            kk, vv = self.k[l][:end], self.v[l][:end]
            blocks = pp.select(q, pos, kk, n_blocks) if n_blocks else None
            o = self.round(pp.attention(q, pos, kk, vv, blocks)[0])
            h = h + o.reshape(M, H * dh) @ w["wo"].T
            b = self.norm(h, w["mlp_norm"])
            g = b @ w["wg"].T
            h = h + self.round(g / (1 + np.exp(-g)) * (b @ w["wu"].T)) @ w["wd"].T
        hn = self.norm(h[-1:], values(self.W["final_norm"], dt))
        return (hn @ values(self.W["lm_head"], dt).T)[0]


def stored_rows(packed, cfg, at):
    import torch
    dt = torch.bfloat16 if cfg["dtype"] == "bf16" else torch.float32
    k = torch.empty((len(at), cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"]), dtype=dt,
                    device="cuda")
    v = torch.empty_like(k)
    packed.read(at, k, v)
    packed.model.synchronize()
    return k.double().cpu().numpy(), v.double().cpu().numpy()


@pytest.mark.parametrize("dtype,dh,n", [("fp32", 64, 300), ("fp32", 128, 256), ("bf16", 64, 300),
                                        ("bf16", 128, 129)])
def test_pack_repair_and_ask(dtype, dh, n):
    if kv is None:
        raise _IMPORT_ERROR
    # A pass differs from the plain decoder by its sums' rounding (fp32: 1e-6 of an entry, bf16:
    # its operands' 2^-9): an entry that lies so near a midpoint of its codes goes to the other
    # one.  Steps are a tenth of an entry or more, so fewer than 1e-4 (2e-2) of the rows' entries
    # do; a pass adds some of the layers before.  Logits take their sum: 1e-3, 2e-2 as without.
    share, tol = (1e-3, 1e-3) if dtype == "fp32" else (6e-2, 2e-2)
    cfg = synth.preset("tiny", dtype=dtype, head_dim=dh, n_heads=4, n_kv_heads=2)
    W = synth.weights(cfg, 0)
    m = kv.Model(cfg, W, max_context=512, max_rows=64)
    doc = synth.document(1, n, cfg["vocab"])
    cache = m.prefill(doc)
    k, v = cache.read(np.arange(n))
    packed = m.pack(cache)
    cache.close()
    assert packed.n == n
    want = pp.stored(k.astype(np.float64)), pp.stored(v.astype(np.float64))
    got = stored_rows(packed, cfg, np.arange(n))
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])

    plain = Plain(cfg, W, *want, cap=n + 64)
    query = synth.fill_tokens(5, 8, cfg["vocab"], cfg["delim_id"])

    def ask(n_blocks):
        before = [x.copy() for x in (plain.k, plain.v)]
        ref = plain.run(query, n + np.arange(8), n_blocks)
        plain.k, plain.v = before  # the query leaves nothing behind
        got = m.packed_logits(packed, query, n_blocks)
        assert np.abs(got - ref).max() <= tol * np.abs(ref).max(), n_blocks
        return got

    dense = ask(0)
    bounds = packed.bounds(1)
    few = ask(2)
    assert not np.array_equal(dense, few)  # two blocks of five
    assert np.array_equal(dense, m.packed_logits(packed, query, 100))
    for a, b in zip(bounds, packed.bounds(1)):
        assert np.array_equal(a, b)
    assert packed.n == n and np.array_equal(stored_rows(packed, cfg, np.arange(n))[0], want[0])

    # an edit: span and scattered positions, in place
    s, new = n // 3, synth.fill_tokens(7, 5, cfg["vocab"], cfg["delim_id"])
    at = np.sort(np.random.default_rng(3).permutation(np.arange(s + 5, n))[:20])
    packed.repair(new, s, at)
    P = np.concatenate([np.arange(s, s + 5), at])
    edited = doc.copy()
    edited[s:s + 5] = new
    plain.run(edited[P], P)
    got = stored_rows(packed, cfg, np.arange(n))
    rest = np.setdiff1d(np.arange(n), P)
    for g, w, old in ((got[0], plain.k, want[0]), (got[1], plain.v, want[1])):
        assert np.array_equal(g[rest], old[rest])  # the others stay
        assert np.mean(g[P] != w[:, P].transpose(1, 0, 2, 3)) <= share
    for l in range(2):
        assert all(np.array_equal(a, b) for a, b in zip(packed.bounds(l), pp.bounds(got[0][:, l])))
    plain.k[:, :n], plain.v[:, :n] = got[0].transpose(1, 0, 2, 3), got[1].transpose(1, 0, 2, 3)
    ask(0)
    ask(2)
    packed.repair([], 0, [])  # nothing
    packed.close()
    m.close()


def test_refusals():
    if kv is None:
        raise _IMPORT_ERROR
    import torch
    cfg = synth.preset("tiny")
    m = kv.Model(cfg, None, max_context=512, max_rows=64)
    doc = synth.document(1, 100, cfg["vocab"])
    cache = m.prefill(doc)
    packed, empty = m.pack(cache), m.packed(10)

    def code(f):
        with pytest.raises(kv.KvrError) as e:
            f()
        return e.value.code
    assert code(lambda: empty.repair([1], 0, [])) == 1
    assert code(lambda: m.packed_logits(empty, [1])) == 1
    assert code(lambda: packed.repair([1], 100, [])) == 2 and code(lambda: packed.repair([1], -1, [])) == 2
    assert code(lambda: packed.repair([-1], 0, [])) == 2
    assert code(lambda: packed.repair([cfg["vocab"]], 0, [])) == 2
    assert code(lambda: packed.repair([1], 5, [5])) == 2 and code(lambda: packed.repair([], 0, [100])) == 2
    assert code(lambda: packed.repair([], 0, [3, 3])) == 2
    assert code(lambda: packed.repair([], 0, np.arange(65))) == 6
    assert code(lambda: m.packed_logits(packed, [])) == 1  # no array, as for logits
    assert code(lambda: m.packed_logits(packed, [1] * 65)) == 2
    assert code(lambda: m.packed_logits(packed, [-1])) == 2
    assert code(lambda: m.packed_logits(packed, [1], -1)) == 2
    assert code(lambda: m.packed_logits(packed, [1], 16385)) == 2
    k = torch.zeros((1, 2, cfg["n_kv_heads"], cfg["head_dim"]), device="cuda")
    packed.write([100], k, k)  # past its tokens
    assert code(lambda: packed.repair([1], 0, [])) == 1
    assert code(lambda: m.packed_logits(packed, [1])) == 1
    cache.close()
    m.close()
    packed.close()  # freed with the model
