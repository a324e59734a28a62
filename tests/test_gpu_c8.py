"""The 8-bit cache against its plain 64-bit form (tests/c8_plain.py): stored values and choices
exactly, attention and weights within the roundings of their types."""
import numpy as np
import pytest
import torch

from paper_2609_17983_gb300 import synth
from tests import c8_plain as cp

try:
    from paper_2609_17983_gb300 import kvrepair as kv
except ImportError as _e:  # pragma: no cover
    kv, _IMPORT_ERROR = None, _e

pytestmark = pytest.mark.gpu

# head size, heads, KV heads: groups of 2, 7 and 9 heads (a tile holds 8 vectors), one
SHAPES = {"dh64": (64, 4, 2), "dh128": (128, 14, 2), "dh128_9": (128, 18, 2), "dh64_1": (64, 3, 3)}
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def models():
    if kv is None:
        raise _IMPORT_ERROR
    made = {}

    def get(shape, dtype, layers=2):
        key = (shape, dtype, layers)
        if key not in made:
            dh, H, G = SHAPES[shape]
            cfg = synth.preset("tiny", dtype=dtype, head_dim=dh, n_heads=H, n_kv_heads=G,
                               n_layers=layers)
            made[key] = kv.Model(cfg, None, seed=0, max_context=256, max_rows=64)
            made[key].set_stream(torch.cuda.current_stream().cuda_stream)
        return made[key]
    yield get
    for m in made.values():
        m.close()


def rows(seed, n, layers, G, dh, dtype, big=0.7):
    """Rows with channels and positions of different sizes, on the GPU."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, layers, G, dh), generator=g)
    x = x * torch.exp(big * torch.randn((G, dh), generator=g))
    x = x * torch.exp(0.5 * torch.randn((n, 1, 1, 1), generator=g))
    return x.to(TORCH[dtype]).cuda()


def f64(t):
    return t.double().cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


class Pair:
    """A cache and its plain form, written alike."""

    def __init__(self, m, shape, dtype, capacity, layers=2):
        self.dh, self.H, self.G = SHAPES[shape]
        self.m, self.dtype, self.L = m, dtype, layers
        self.c = m.cache8(capacity)
        self.plain = [[cp.Head(self.dh) for _ in range(self.G)] for _ in range(layers)]

    def write(self, at, k, v, l0=0, l1=None):
        l1 = self.L if l1 is None else l1
        self.c.write(at, k, v, layer_begin=l0, layer_end=l1)
        kd, vd = f64(k), f64(v)
        for l in range(l0, l1):
            for g in range(self.G):
                self.plain[l][g].write(at, kd[:, l - l0, g], vd[:, l - l0, g])

    def fill(self, seed, n, start=0, size=1.0):
        k = rows(seed, n, self.L, self.G, self.dh, self.dtype) * size
        v = rows(seed + 1, n, self.L, self.G, self.dh, self.dtype) * size
        self.write(np.arange(start, start + n), k, v)
        return self

    def keep(self, kept):
        for l in range(self.L):
            for g in range(self.G):
                self.plain[l][g].keep(kept[l][g])

    def check(self, cache=None, l0=0, l1=None):
        """Everything that the cache holds."""
        c, l1 = cache or self.c, self.L if l1 is None else l1
        n = len(self.plain[l0][0].k)
        k = torch.empty((n, l1 - l0, self.G, self.dh), dtype=TORCH[self.dtype], device="cuda")
        v = torch.empty_like(k)
        number = torch.full((l1 - l0, self.G, n), 77, dtype=torch.int32, device="cuda")
        weight = torch.full((l1 - l0, self.G, n), 77.0, device="cuda")
        c.read(np.arange(n), k, v, layer_begin=l0, layer_end=l1)
        c.entries(number, weight, layer_begin=l0, layer_end=l1)
        k, v = f64(k), f64(v)
        for l in range(l0, l1):
            for g in range(self.G):
                p = self.plain[l][g]
                wk, wv = p.read()
                assert same(k[:, l - l0, g], wk) and same(v[:, l - l0, g], wv), (l, g)
                assert np.array_equal(number[l - l0, g].cpu().numpy(), p.number)
                assert np.array_equal(f64(weight[l - l0, g]), p.weight, equal_nan=True)


# ------------------------------------------------------------------ rows

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", ["dh64", "dh128"])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 200])
def test_store(models, shape, dtype, n):
    m = models(shape, dtype)
    p = Pair(m, shape, dtype, n + 70)
    p.fill(n, n)
    assert p.c.n == n
    p.check()
    # scattered entries of one layer, in place, larger than the rest: powers rise there alone
    at = np.unique(np.r_[0, n // 3, n // 2, n - 1])
    k2, v2 = rows(5, len(at), 1, p.G, p.dh, dtype) * 9, rows(6, len(at), 1, p.G, p.dh, dtype)
    p.write(at, k2, v2, l0=1)
    p.check()
    # smaller again: powers stay where other entries do
    p.write(at, k2 / 64, v2 / 64, l0=1)
    p.check()
    # appended behind, two blocks at once where they end, and far larger
    p.fill(7, 5, n, 100.0)
    p.fill(9, 65, n + 5, 0.01)
    assert p.c.n == n + 70
    p.check()
    p.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_store_edges_of_the_grid(models, dtype):
    """Ties of codes, borders of the powers, zeros, the least and largest powers, NaN, infinity."""
    dh, H, G = SHAPES["dh64"]
    m = models("dh64", dtype)
    mid = torch.tensor((cp.VALUES[1:] + cp.VALUES[:-1]) / 2)  # 7 bits: exact in both types
    for case, size in enumerate([1.0, 2.0 ** -40, 2.0 ** 100, 2.0 ** -100, 2.0 ** -108]):
        x = torch.zeros((70, 2, G, dh), dtype=torch.float64)
        x[0, :, :, :63], x[1, :, :, :63] = mid[:63], -mid[63:]
        x[2, :, :, 0] = 448.0
        x[3, 0, :, 0] = 450.0  # above the border: the power doubles in layer 0
        x[64, 0, :, 0], x[64, 1, :, 0] = 448.0, 449.0
        x[65] = 2.0 ** -10
        x = (x * size).to(TORCH[dtype])
        p = Pair(m, "dh64", dtype, 70)
        p.write(np.arange(70), x.cuda(), x.flip(0).contiguous().cuda())
        p.check()
        p.c.close()
    x = torch.zeros((64, 2, G, dh))
    p = Pair(m, "dh64", dtype, 64)
    p.write(np.arange(64), x.to(TORCH[dtype]).cuda(), x.to(TORCH[dtype]).cuda())
    p.check()
    x[:] = torch.randn(x.shape, generator=torch.Generator().manual_seed(1))
    x[32, :, :, 0], x[33, 0, 0, 63], x[34, 1, 1, 5], x[35, :, 1, 0] = 3e38, float("nan"), float(
        "inf"), -float("inf")
    x[36] = 1e-39  # below the normal numbers
    x[37, :, 0, 1], x[38, :, :, 2] = 248 * 2.0 ** 120, 247 * 2.0 ** 120  # marked, and the largest
    x = x.to(TORCH[dtype])
    p.write(np.arange(64), x.cuda(), x.flip(0).contiguous().cuda())
    p.check()
    p.write([33, 34], torch.ones((2, 2, G, dh), dtype=TORCH[dtype]).cuda(),
            torch.ones((2, 2, G, dh), dtype=TORCH[dtype]).cuda())  # marks go with their rows
    p.check()
    p.c.close()


@pytest.mark.parametrize("shape,dtype", [("dh128", "bf16"), ("dh64", "fp32")])
def test_store_many_scattered_rows(models, shape, dtype):
    """More scattered entries than come with a launch, some blocks whole, a NaN among them."""
    m = models(shape, dtype)
    n = 64 * 20 - 7
    p = Pair(m, shape, dtype, n).fill(1, n)
    at = np.unique(np.r_[np.arange(0, n, 2), np.arange(128, 192)])
    k = rows(3, len(at), 2, p.G, p.dh, dtype) * 3
    v = rows(4, len(at), 2, p.G, p.dh, dtype)
    k[100, 1, 0, 3] = float("nan")
    p.write(at, k, v)
    p.check()
    out = torch.empty((len(at), 1, p.G, p.dh), dtype=TORCH[dtype], device="cuda")
    vout = torch.empty_like(out)
    p.c.read(at, out, vout, layer_begin=1)  # a list that is sent
    for g in range(p.G):
        wk, wv = p.plain[1][g].read()
        assert same(f64(out)[:, 0, g], wk[at]) and same(f64(vout)[:, 0, g], wv[at])
    p.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", ["dh64", "dh128"])
def test_read_into_arrays_of_any_alignment(models, shape, dtype):
    """16 bytes past a boundary of 32, one of the two or both, nothing beside them touched; and a
    list of entries beside a run."""
    m = models(shape, dtype)
    p = Pair(m, shape, dtype, 150).fill(3, 150)
    for at in (np.arange(20, 150), np.r_[0, 5, 63, 64, 149]):
        wide = torch.empty((2, len(at), 2, p.G, p.dh), dtype=TORCH[dtype], device="cuda")
        p.c.read(at, wide[0], wide[1])
        want = [np.stack([np.stack([p.plain[l][g].read()[kv_][at] for g in range(p.G)], 1)
                          for l in range(2)], 1) for kv_ in range(2)]
        assert same(f64(wide[0]), want[0]) and same(f64(wide[1]), want[1])
        off, n = 16 // wide.element_size(), wide[0].numel()
        for k_off, v_off in ((off, 0), (0, off), (off, 3 * off)):
            flat = torch.full((2, n + 8 * off), 77.0, dtype=TORCH[dtype], device="cuda")
            into = [flat[i, o:o + n] for i, o in enumerate((k_off, v_off))]
            p.c.read(at, *[x.view(wide[0].shape) for x in into])
            for i, o in enumerate((k_off, v_off)):
                assert torch.equal(flat[i, o:o + n], wide[i].reshape(-1))
                assert (flat[i, :o] == 77).all() and (flat[i, o + n:] == 77).all()


def test_layers_of_different_lengths(models):
    """A step appends layer by layer; what a layer does not hold yet is refused or left alone."""
    m = models("dh64", "bf16", 4)
    p = Pair(m, "dh64", "bf16", 200, 4).fill(1, 100)
    one = [rows(s, 1, 1, p.G, p.dh, "bf16") for s in (3, 4)]
    for l in range(4):
        assert p.c.n == 100
        p.write([100], one[0], one[1], l, l + 1)
        p.check(l0=l, l1=l + 1)
        if l < 3:
            with pytest.raises(kv.KvrError) as e:
                p.c.choose(torch.empty((4, p.G, 5), dtype=torch.int32, device="cuda"))
            assert e.value.code == 1
            with pytest.raises(kv.KvrError) as e:
                p.c.entries(torch.empty((4, p.G, 101), dtype=torch.int32, device="cuda"))
            assert e.value.code == 2
    assert p.c.n == 101
    p.write([101], one[0], one[1], 2, 3)
    two = [rows(s, 3, 4, p.G, p.dh, "bf16") for s in (5, 6)]
    p.write([50, 101, 102], two[0], two[1])  # new to three layers, rewritten in one
    p.check()
    assert p.c.n == 103
    p.c.close()


# ------------------------------------------------------------------ attention and weights

def queries(seed, R, H, dh, dtype, size=1.5):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn((R, H, dh), generator=g)).to(TORCH[dtype]).cuda()


def score_error(smax):
    """How far a score's exponential may be off, relatively: 2^-19 for the exponential itself and
    the roundings of its argument next to a reference of up to 2^5, and 16 additions and products
    (an fp32 model's q to 22 bits among them) each off by at most 2^-23 of the sum of magnitudes."""
    return 2.0 ** -19 + 16 * 2.0 ** -23 * smax


def out_bound(dtype, ref, vmax, smax):
    """bf16: the output to 8 bits, the weights to 11 (so 2^-11 of the largest value at most); fp32:
    24 and 22.  A score's error moves its weight by as much, the sum by as much again."""
    delta = 2 * score_error(smax)
    if dtype == "bf16":
        return 2.0 ** -8 * np.abs(ref) + ((2.0 ** -11 + delta) * vmax)[..., None]
    return 2.0 ** -24 * np.abs(ref) + ((2.0 ** -22 + delta) * vmax)[..., None]


def check_attention(p, layer, q, seen, out, weight=None, old=None, decay=0.0):
    q, got = f64(q), f64(out)
    grp = p.H // p.G
    for g in range(p.G):
        k, v = p.plain[layer][g].read()
        hs = slice(g * grp, (g + 1) * grp)
        ref, w, vmax, smax = cp.attention(q[:, hs], seen, k, v)
        assert np.array_equal(np.isnan(got[:, hs]), np.isnan(ref))
        err = np.abs(got[:, hs] - ref) - out_bound(p.dtype, ref, vmax, smax)
        assert not (err > 0).any(), float(np.nanmax(err))
        if weight is None:
            continue
        total = cp.summed(w)
        # numerator and sum each by a score's error, and by another for the logarithm of the sum;
        # R * heads additions; the old weight's product and sum
        part = cp.summed(np.where(np.isfinite(w), w, np.nan) * (3 * score_error(smax))[..., None])
        was = 0.0 if not decay else decay * old[g]
        lim = part + (len(q) * grp + 2) * 2.0 ** -24 * (total + np.abs(was)) + 2.0 ** -120
        err = np.abs(f64(weight[g]) - (was + total)) - lim
        assert not (err > 0).any(), float(err.max())


def weights_of(c, layer, n, G):
    w = torch.full((1, G, n), 77.0, device="cuda")
    if n:
        c.entries(None, w, layer_begin=layer, layer_end=layer + 1)
    return w[0]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("n,R", [(1, 1), (64, 1), (65, 3), (500, 1), (1000, 13)])
def test_attention_one_document(models, shape, dtype, n, R):
    m = models(shape, dtype)
    p = Pair(m, shape, dtype, n + 3).fill(n, n)
    seen = np.sort(np.random.default_rng(R).integers(-1, n, R))
    seen[-1] = n - 1
    r = m.rows8([(p.c, seen)])
    q = queries(n + R, R, p.H, p.dh, dtype)
    out, again = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
    r.attention(1, q, out)
    check_attention(p, 1, q, seen, out)
    r.attention(1, q, again, weigh=0.0)
    assert torch.equal(out, again)
    first = weights_of(p.c, 1, n, p.G)
    check_attention(p, 1, q, seen, again, first)
    r.attention(1, q, again, weigh=0.5)
    check_attention(p, 1, q, seen, again, weights_of(p.c, 1, n, p.G), f64(first), 0.5)
    assert not weights_of(p.c, 0, n, p.G).any()  # the other layer's are as they were
    r.close()
    p.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_several_documents_and_moves(models, dtype):
    m = models("dh128", dtype)
    lens = [1, 2, 300, 129, 64]
    docs = [Pair(m, "dh128", dtype, n + 3).fill(10 * i + 3, n) for i, n in enumerate(lens)]
    seen = [[-1], [-1, 0], [5, 5, 299], [], [0, 63]]
    r = m.rows8([(d.c, s) for d, s in zip(docs, seen)])
    q = queries(1, r.n, 14, 128, dtype)
    docs[3].c.set_weights(torch.full((2, 2, 129), 3.0, device="cuda"))
    for move in range(2):
        if move:
            seen = [[0], [0, 0], [0, 130, 131], [], [-1, -1]]
            r.move(np.concatenate(seen).astype(np.int32))
        out = torch.full_like(q, float("nan"))
        old = [f64(weights_of(d.c, 0, n, 2)) for d, n in zip(docs, lens)]
        r.attention(0, q, out, weigh=1.0)
        i = 0
        for d, s, n, o in zip(docs, seen, lens, old):
            if s:
                check_attention(d, 0, q[i:i + len(s)], s, out[i:i + len(s)],
                                weights_of(d.c, 0, n, 2), o, 1.0)
            i += len(s)
        assert (weights_of(docs[3].c, 0, 129, 2) == 3).all()  # no rows: its weights stay
    r.close()


@pytest.mark.parametrize("shape,dtype,n,R,spread", [
    ("dh64", "bf16", 4000, 1201, True), ("dh128", "bf16", 2000, 300, False),
    ("dh128", "bf16", 2049, 501, True), ("dh64", "fp32", 700, 400, False)])
def test_attention_many_rows(models, shape, dtype, n, R, spread):
    """Odd lengths, rows that see nothing, a second document with few rows, q rows apart, marks."""
    m = models(shape, dtype)
    p = Pair(m, shape, dtype, n + 1)
    k, v = rows(n, n, 2, p.G, p.dh, dtype), rows(n + 1, n, 2, p.G, p.dh, dtype)
    k[n - 10, :, 0, 7], v[n - 5, :, p.G - 1, 3] = float("nan"), float("inf")
    p.write(np.arange(n), k, v)
    small = Pair(m, shape, dtype, 100).fill(5, 100)
    seen = np.linspace(0, n - 1, R).astype(int) if spread else np.arange(n - R, n)
    seen[:3] = -1
    r = m.rows8([(small.c, [50]), (p.c, seen)])
    wide = torch.randn((R + 1, p.H + 2 * p.G, p.dh), device="cuda").to(TORCH[dtype])
    q = wide[:, :p.H]
    out = torch.full((R + 1, p.H, p.dh), float("nan"), dtype=TORCH[dtype], device="cuda")
    r.attention(1, q, out, weigh=0.0)
    check_attention(small, 1, q[:1], [50], out[:1], weights_of(small.c, 1, 100, p.G))
    check_attention(p, 1, q[1:], seen, out[1:], weights_of(p.c, 1, n, p.G))
    assert (out[1:4] == 0).all()
    again = torch.empty_like(out)
    r.attention(1, q.contiguous(), again)
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(again))
    r.close()
    p.c.close()


@pytest.mark.parametrize("rows_,last", [(3, 130), (200, 300), (200, 1800), (1300, 700)])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_weights_behind_the_last_row(models, rows_, last, decay):
    """Entries past the last one that any row sees, by all ways of taking the weights: theirs decay
    and get nothing, those of other layers stay."""
    m, n = models("dh128", "bf16"), 2111
    p = Pair(m, "dh128", "bf16", n + 70).fill(21, n)
    old = torch.rand((2, p.G, n), generator=torch.Generator().manual_seed(4)).cuda()
    p.c.set_weights(old)
    seen = np.linspace(0, last, rows_).astype(int)
    r = m.rows8([(p.c, seen)])
    q = queries(22, rows_, p.H, p.dh, "bf16")
    out = torch.empty_like(q)
    r.attention(1, q, out, weigh=decay)
    got = weights_of(p.c, 1, n, p.G)
    check_attention(p, 1, q, seen, out, got, f64(old[1]), decay)
    assert torch.equal(torch.as_tensor(got)[:, last + 1:].cpu().float(),
                       (old[1] * decay)[:, last + 1:].cpu())
    left = torch.empty((1, p.G, n), device="cuda")
    p.c.entries(None, left, layer_begin=0, layer_end=1)
    assert torch.equal(left[0], old[0])
    r.close()
    p.c.close()


def test_attention_rows_apart_sizes_and_streams(models):
    """Queries of very different sizes; blocks whose powers differ; a stream of its own."""
    m = models("dh128", "bf16")
    p = Pair(m, "dh128", "bf16", 400).fill(3, 200)
    p.fill(5, 100, 200, 2.0 ** -12)
    p.fill(7, 100, 300, 8.0)
    seen = np.array([10, 250, 399])
    r = m.rows8([(p.c, seen)])
    wide = torch.randn((3, p.H + 2 * p.G, p.dh), device="cuda").bfloat16()
    wide[0] *= 1e-6
    wide[2] *= 0.5
    wide[1, 0, 5:] *= 2.0 ** -30  # entries of one vector far apart
    q = wide[:, :p.H]
    out = torch.empty((3, p.H, p.dh), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    m.set_stream(s.cuda_stream)
    r.attention(1, q, out, weigh=0.0)
    m.synchronize()
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    check_attention(p, 1, q, seen, out, weights_of(p.c, 1, 400, p.G))
    r.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_not_finite(models, dtype):
    """A marked entry, or a query that is not finite, reaches the rows that see it alone, and their
    weights nothing."""
    m = models("dh128", dtype)
    n = 200
    p = Pair(m, "dh128", dtype, n)
    k, v = rows(1, n, 2, p.G, p.dh, dtype), rows(2, n, 2, p.G, p.dh, dtype)
    k[100, :, 0, 7] = float("nan")
    v[130, :, 1, 3] = float("inf")
    p.write(np.arange(n), k, v)
    seen = np.array([50, 99, 100, 129, 130, 199])
    r = m.rows8([(p.c, seen)])
    q = queries(4, len(seen), p.H, p.dh, dtype)
    q[1, 3, 5], q[0, 9, 0] = float("nan"), float("inf")
    out = torch.empty_like(q)
    p.c.set_weights(torch.full((2, p.G, n), float("nan"), device="cuda"))
    r.attention(0, q, out, weigh=0.0)  # a factor of zero forgets even that
    check_attention(p, 0, q, seen, out, weights_of(p.c, 0, n, p.G))
    got = f64(out).reshape(len(seen), p.G, -1)
    assert np.isnan(got[2:]).all(2).tolist() == [[True, False], [True, False], [True, True],
                                                 [True, True]]
    bad = np.isnan(f64(out)).any(2)
    assert bad[1].tolist() == [h == 3 for h in range(p.H)]
    assert bad[0].tolist() == [h == 9 for h in range(p.H)]
    r.close()


@pytest.mark.parametrize("dtype,rows_", [("bf16", 3), ("fp32", 3), ("bf16", 200), ("bf16", 1500)])
def test_zero_queries_and_tiny_keys(models, dtype, rows_):
    """Products that vanish leave equal weights to the entries that a row sees."""
    m = models("dh64", dtype)
    n = 1600
    p = Pair(m, "dh64", dtype, n)
    k = torch.full((n, 2, p.G, p.dh), 2.0 ** -120, dtype=TORCH[dtype], device="cuda")
    k[:, 1] = 0.0
    v = rows(3, n, 2, p.G, p.dh, dtype)
    p.write(np.arange(n), k, v)
    seen = np.linspace(0, n - 1, rows_).astype(int)
    r = m.rows8([(p.c, seen)])
    q = queries(4, rows_, p.H, p.dh, dtype)
    q[::2] = 0.0
    q[1::2] *= 2.0 ** -110
    for layer in range(2):
        out = torch.full_like(q, float("nan"))
        r.attention(layer, q, out, weigh=0.0)
        check_attention(p, layer, q, seen, out, weights_of(p.c, layer, n, p.G))
    r.close()


@pytest.mark.parametrize("rows_", [40, 300, 1100])
def test_blocks_of_different_powers(models, rows_):
    """Blocks 2^20 apart beside one another, by few rows and many."""
    m = models("dh128", "bf16")
    n = 1500
    p = Pair(m, "dh128", "bf16", n)
    k, v = rows(1, n, 2, p.G, p.dh, "bf16"), rows(2, n, 2, p.G, p.dh, "bf16")
    for b in range(0, n, 64):
        k[b:b + 64] *= 2.0 ** -(b // 64 % 7)
        v[b:b + 64] *= 2.0 ** (10 - 10 * (b // 64 % 3))
    p.write(np.arange(n), k, v)
    seen = np.linspace(3, n - 1, rows_).astype(int)
    r = m.rows8([(p.c, seen)])
    q = queries(4, rows_, p.H, p.dh, "bf16")
    out = torch.empty_like(q)
    r.attention(0, q, out, weigh=0.0)
    check_attention(p, 0, q, seen, out, weights_of(p.c, 0, n, p.G))
    r.close()


def test_weights_of_several_launches(models):
    """More scores than a launch's scratch holds, an earlier weight's factor applied once."""
    m = models("dh64", "fp32", 1)
    n, R = 4500, 1500  # 375 tiles of 2 KV heads over 3750 keys on average: 90 MB
    p = Pair(m, "dh64", "fp32", n, 1).fill(5, n)
    small = Pair(m, "dh64", "fp32", 70, 1).fill(7, 70)
    seen = np.arange(n - R, n)
    r = m.rows8([(p.c, seen), (small.c, [3, 69])])
    q = queries(6, R + 2, p.H, p.dh, "fp32")
    out = torch.empty_like(q)
    p.c.set_weights(torch.full((1, p.G, n), 8.0, device="cuda"))
    small.c.set_weights(torch.full((1, p.G, 70), 4.0, device="cuda"))
    before = m.launches()
    r.attention(0, q, out, weigh=0.25)
    assert m.launches() - before >= 4
    check_attention(p, 0, q[:R], seen, out[:R], weights_of(p.c, 0, n, p.G),
                    np.full((p.G, n), 8.0), 0.25)
    check_attention(small, 0, q[R:], [3, 69], out[R:], weights_of(small.c, 0, 70, p.G),
                    np.full((p.G, 70), 4.0), 0.25)
    r.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_values_of_many_entries(models, dtype):
    """Values near the types' largest, in sums of equal weights: nothing overflows on the way."""
    m = models("dh64", dtype)
    n = 3000
    p = Pair(m, "dh64", dtype, n)
    k = torch.zeros((n, 2, p.G, p.dh), dtype=TORCH[dtype], device="cuda")
    v = torch.full_like(k, 2.9e38)
    v[::3] = -2.9e38
    p.write(np.arange(n), k, v)
    r = m.rows8([(p.c, [n - 1])])
    q = queries(1, 1, p.H, p.dh, dtype)
    out = torch.empty_like(q)
    r.attention(0, q, out, weigh=0.0)
    check_attention(p, 0, q, [n - 1], out, weights_of(p.c, 0, n, p.G))
    r.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,step", [(20011, 3), (70000, 7)])
def test_long_documents(models, dtype, n, step):
    """Parts that meet through memory; one key that takes most of the weight."""
    m = models("dh64", dtype, 1)
    p = Pair(m, "dh64", dtype, n, 1)
    k, v = rows(1, n, 1, p.G, p.dh, dtype), rows(2, n, 1, p.G, p.dh, dtype)
    q = queries(3, 3, p.H, p.dh, dtype)
    k[n // step, 0, 0] = (q[1, 0] * 2).to(k.dtype)
    p.write(np.arange(n), k, v)
    seen = [n // 2, n - 2, n - 1]
    r = m.rows8([(p.c, seen)])
    out = torch.empty_like(q)
    for _ in range(2):
        r.attention(0, q, out, weigh=0.0)
    check_attention(p, 0, q, seen, out, weights_of(p.c, 0, n, p.G))
    first = weights_of(p.c, 0, n, p.G)
    again = torch.empty_like(out)
    r.attention(0, q, again, weigh=0.0)
    assert torch.equal(out, again) and torch.equal(first, weights_of(p.c, 0, n, p.G))
    r.close()
    p.c.close()


# ------------------------------------------------------------------ eviction

@pytest.mark.parametrize("n,keep,first,recent", [
    (1, 1, 0, 0), (2, 1, 0, 0), (64, 30, 0, 0), (65, 64, 4, 30), (500, 250, 4, 32), (1025, 1, 0, 1),
    (3000, 2999, 0, 0), (3000, 3000, 0, 0), (3000, 900, 900, 0), (5000, 1700, 16, 128)])
def test_choice(models, n, keep, first, recent):
    m = models("dh64", "bf16")
    p = Pair(m, "dh64", "bf16", n).fill(1, n)
    rng = np.random.default_rng(n + keep)
    for kind in range(3):
        w = np.exp(2 * rng.normal(size=(2, p.G, n))).astype(np.float32)
        if kind == 1:  # many ties, zeros of both signs, negative ones, infinities and NaN
            w = rng.integers(-2, 3, (2, p.G, n)).astype(np.float32)
            w[rng.random(w.shape) < 0.1] = -0.0
            w[rng.random(w.shape) < 0.05] = np.nan
            w[rng.random(w.shape) < 0.02] = np.inf
            w[rng.random(w.shape) < 0.02] = -np.inf
        if kind == 2:
            w[:] = 1.0
        p.c.set_weights(torch.from_numpy(w).cuda())
        kept = torch.full((2, p.G, keep), -5, dtype=torch.int32, device="cuda")
        p.c.choose(kept, first=first, recent=recent)
        for l in range(2):
            for g in range(p.G):
                want = cp.choose(w[l, g], keep, first, recent)
                assert np.array_equal(kept[l, g].cpu().numpy(), want), kind
    p.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", ["dh64", "dh128"])
@pytest.mark.parametrize("n,keep", [(1, 1), (64, 1), (130, 64), (130, 65), (1000, 300),
                                    (1500, 1400), (500, 500), (200, 0)])
def test_keep(models, shape, dtype, n, keep):
    """Entries of blocks of different powers, marked ones among them, into another cache and in
    place; then appended to."""
    m = models(shape, dtype)
    p = Pair(m, shape, dtype, n + 70)
    k, v = rows(n, n, 2, SHAPES[shape][2], SHAPES[shape][0], dtype), rows(
        n + 1, n, 2, SHAPES[shape][2], SHAPES[shape][0], dtype)
    size = torch.exp2(torch.randint(-12, 12, (n, 1, 1, 1), generator=torch.Generator().manual_seed(n)))
    k, v = (k * size.cuda()).to(k.dtype), (v / size.cuda()).to(v.dtype)
    k[n // 2, 1, 0, 0] = float("nan")
    p.write(np.arange(n), k, v)
    w = torch.rand((2, p.G, n), generator=torch.Generator().manual_seed(1)).cuda()
    p.c.set_weights(w)
    for l in range(2):
        for g in range(p.G):
            p.plain[l][g].weight = f64(w[l, g])
    p.check()
    kept = torch.empty((2, p.G, keep), dtype=torch.int32, device="cuda")
    p.c.choose(kept, first=min(keep, 1))
    other = Pair(m, shape, dtype, keep + 9)
    other.fill(3, keep + 9)  # what it held goes
    p.c.keep(kept, into=other.c)
    assert p.c.n == n and other.c.n == keep
    p.check()
    p.keep(kept.cpu().numpy())
    if keep:
        p.check(other.c)
    p.c.keep(kept)
    assert p.c.n == keep
    if keep:
        p.check()
    p.fill(11, 70, keep)
    p.check()
    assert p.plain[0][0].number[-1] == n + 69
    p.c.close()
    other.c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", ["dh64", "dh128"])
@pytest.mark.parametrize("e", [27, 28, 40, 119])
def test_keep_zeros_of_large_powers(models, shape, dtype, e):
    """Two blocks whose entries were rounded to zero under one magnitude each, K's in one layer and
    V's in the other; that magnitude dropped, so that zeros move to the least power or beside tiny
    entries.  They stay zeros, into another cache and in place, and attention is finite."""
    m, n = models(shape, dtype), 200
    p = Pair(m, shape, dtype, n)
    k, v = (rows(s, n, 2, p.G, p.dh, dtype) for s in (41, 42))
    for x, l in ((k, 0), (v, 1)):
        x[[5, 70], l, :, 3] = 448 * 2.0 ** e  # the block's power is 2^e
        x[128:, l] *= 2.0 ** -60
    p.write(np.arange(n), k, v)
    p.check()
    at = np.setdiff1d(np.arange(n), [5, 70])
    kept = torch.as_tensor(at, dtype=torch.int32).repeat(2, p.G, 1).cuda()
    other = m.cache8(len(at))
    p.c.keep(kept, into=other)
    p.keep(kept.cpu().numpy())
    assert not p.plain[0][0].k[:120].any() and not p.plain[1][0].v[:120].any()
    p.check(other)
    p.c.keep(kept)
    p.check()
    seen = np.array([3, 63, 100, len(at) - 1])
    r = m.rows8([(p.c, seen)])
    q = queries(43, len(seen), p.H, p.dh, dtype)
    out = torch.empty_like(q)
    for l in range(2):
        r.attention(l, q, out, weigh=0.0)
        assert torch.isfinite(out).all()
        check_attention(p, l, q, seen, out, weights_of(p.c, l, len(at), p.G))
    r.close()
    other.close()
    p.c.close()


def test_keep_lists_of_the_caller(models):
    """Entries outside the cache or out of order are kept as zeros that have no number."""
    m = models("dh64", "bf16")
    n = 300
    p = Pair(m, "dh64", "bf16", n).fill(1, n)
    lists = torch.arange(0, 200, dtype=torch.int32).repeat(2, p.G, 1) + 100
    lists[0, 0, 5], lists[0, 1, 70] = 300, -1
    lists[1, 0, 100:103] = torch.tensor([250, 250, 10])
    lists[1, 1, 3] = 2 ** 31 - 1
    bad = {(0, 0): [5], (0, 1): [70], (1, 0): [101, 102], (1, 1): [3, 4]}
    bad[(0, 0)].append(6)  # 300 before it is larger
    for into in (m.cache8(200), None):
        want = [[np.array(p.plain[l][g].k) for g in range(p.G)] for l in range(2)]
        p.c.keep(lists.cuda(), into=into)
        c = into or p.c
        number = torch.empty((2, p.G, 200), dtype=torch.int32, device="cuda")
        weight = torch.empty((2, p.G, 200), device="cuda")
        c.entries(number, weight)
        k = torch.empty((200, 2, p.G, p.dh), dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        c.read(np.arange(200), k, v)
        for l in range(2):
            for g in range(p.G):
                for i in range(200):
                    gone = i in bad[(l, g)]
                    gone = gone or (l, g) == (1, 0) and i > 102 and lists[l, g, i] <= lists[l, g, i - 1]
                    e = int(lists[l, g, i])
                    assert int(number[l, g, i]) == (-1 if gone else e), (l, g, i)
                    if gone:
                        assert not f64(k[i, l, g]).any() and not f64(v[i, l, g]).any()
                    else:
                        assert same(f64(k[i, l, g]), want[l][g][e])
    p.c.close()


def test_long_document_in_place(models):
    """More blocks than a cluster's CTAs take in a round."""
    m = models("dh64", "fp32", 1)
    n, keep = 9000, 8000
    p = Pair(m, "dh64", "fp32", n, 1).fill(1, n)
    w = torch.rand((1, p.G, n), generator=torch.Generator().manual_seed(2)).cuda()
    p.c.set_weights(w)
    kept = torch.empty((1, p.G, keep), dtype=torch.int32, device="cuda")
    p.c.choose(kept)
    p.c.keep(kept)
    for g in range(p.G):
        p.plain[0][g].weight = f64(w[0, g])
    p.keep(kept.cpu().numpy())
    p.check()
    p.c.close()


def test_a_million_entries():
    """The largest cache: blocks past 2^32 bytes, one row and many, its weights, a choice, and what is
    kept of it.  The reference on the GPU, in 64 bits."""
    if kv is None:
        raise _IMPORT_ERROR
    n, L, G, H, dh, at = 1 << 20, 3, 8, 16, 128, 1 << 17
    m = kv.Model(synth.preset("tiny", dtype="bf16", head_dim=dh, n_heads=H, n_kv_heads=G, n_layers=L),
                 None, seed=0, max_context=256, max_rows=64)
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    c = m.cache8(n)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(0, n, at):
        k, v = (torch.randn((at, L, G, dh), generator=gen, device="cuda", dtype=torch.bfloat16)
                for _ in range(2))
        c.write(np.arange(i, i + at), k, v)
    assert c.n == n
    del k, v
    k, v = (torch.empty((n, 1, G, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.read(np.arange(n), k, v, layer_begin=2)
    for rows_ in (1, 70):
        seen = np.sort(np.r_[n - 1, np.arange(n - rows_, n - 1) - 997 * np.arange(rows_ - 1)])
        r = m.rows8([(c, seen)])
        q = queries(rows_, rows_, H, dh, "bf16", 2.0)
        out = torch.empty_like(q)
        r.attention(2, q, out, weigh=0.0)
        weight = torch.empty((1, G, n), device="cuda")
        c.entries(None, weight, layer_begin=2)
        last = torch.as_tensor(seen, device="cuda").repeat_interleave(H // G)[:, None]
        masked = torch.arange(n, device="cuda")[None] > last
        for g in range(G):
            kg, vg = k[:, 0, g].double(), v[:, 0, g].double()
            qg = q[:, g * (H // G):(g + 1) * (H // G)].reshape(-1, dh).double()
            x = (qg @ kg.T / dh ** 0.5).masked_fill(masked, -float("inf"))
            w = torch.softmax(x, -1)
            smax = f64((qg.abs() @ kg.abs().T / dh ** 0.5).amax(-1))
            ref = f64(w @ vg)
            got = f64(out[:, g * (H // G):(g + 1) * (H // G)].reshape(-1, dh))
            # the softmax's sum: no more than n / 64 additions one after another (a launch's parts
            # fill the chip, in each two threads or more a vector with four sums each)
            adds = n / 64 * 2.0 ** -24
            lim = out_bound("bf16", ref, float(vg.abs().max()) * np.ones(len(ref)), smax)
            assert (np.abs(got - ref) <= lim + 2 * adds * np.abs(ref)).all()
            total = w.sum(0)
            part = (w * torch.as_tensor(3 * score_error(smax) + adds, device="cuda")[:, None]).sum(0)
            err = (weight[0, g].double() - total).abs() - part - (len(ref) + 2) * 2.0 ** -24 * total
            assert float(err.max()) <= 2.0 ** -120
            del x, w, total, part, err, kg
        r.close()
    # distinct weights: the choice is known
    w = torch.stack([torch.randperm(n, generator=gen, device="cuda") for _ in range(L * G)]).float()
    c.set_weights(w.view(L, G, n))
    keep = 1000
    kept = torch.empty((L, G, keep), dtype=torch.int32, device="cuda")
    c.choose(kept, first=4, recent=32)
    w[:, :4] = w[:, n - 32:] = float("inf")
    want = torch.topk(w, keep, -1).indices.sort(-1).values.view(L, G, keep)
    assert torch.equal(kept.long(), want)
    into = m.cache8(keep)
    c.keep(kept, into=into)
    number = torch.empty_like(kept)
    into.entries(number)
    assert torch.equal(number, kept)
    k2, v2 = (torch.empty((keep, 1, G, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    into.read(np.arange(keep), k2, v2, layer_begin=2)
    for full, some in ((k, k2), (v, v2)):
        old = torch.gather(full[:, 0], 0, want[2].T[:, :, None].expand(-1, -1, dh)).double()
        # a block's new power may be larger: half a step of 4 bits, or of the least code under it
        lim = 2.0 ** -4 * old.abs() + 2.0 ** -10 * 2.0 ** -6
        assert ((some[:, 0].double() - old).abs() <= lim).all()
    m.close()


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_document_shortened_while_it_grows(models, dtype):
    """Steps as a decoding program makes them: each layer's row appended, attended to and weighed;
    every 40 steps the cache is cut back to 100 entries in place."""
    m = models("dh128", dtype)
    p = Pair(m, "dh128", dtype, 160).fill(1, 120)
    H, G, dh = p.H, p.G, p.dh
    r = m.rows8([(p.c, [119])])
    for step in range(100):
        e = len(p.plain[0][0].k)
        r.move([e])
        for l in range(2):
            k, v = rows(1000 + 2 * step + l, 1, 1, G, dh, dtype), rows(7 + step, 1, 1, G, dh, dtype)
            p.write([e], k, v, l, l + 1)
            q = queries(3000 + 2 * step + l, 1, H, dh, dtype)
            out = torch.empty_like(q)
            r.attention(l, q, out, weigh=0.9)
            old = [np.r_[p.plain[l][g].weight[:e], 0.0] for g in range(G)]
            w = weights_of(p.c, l, e + 1, G)
            check_attention(p, l, q, [e], out, w, old, 0.9)
            for g in range(G):
                p.plain[l][g].weight = f64(w[g])
        if step % 40 == 39:
            kept = torch.empty((2, G, 100), dtype=torch.int32, device="cuda")
            p.c.choose(kept, first=4, recent=20)
            for l in range(2):
                for g in range(G):
                    want = cp.choose(p.plain[l][g].weight, 100, 4, 20)
                    assert np.array_equal(kept[l, g].cpu().numpy(), want)
            p.c.keep(kept)
            p.keep(kept.cpu().numpy())
            p.check()
    assert p.plain[0][0].number[-1] == 219
    p.check()
    r.close()


def test_captured_and_replayed():
    """Attention with weights in a CUDA graph, beside eager calls of larger rows in between, which
    outgrow the scratch that the graph holds; what cannot be captured is refused."""
    if kv is None:
        raise _IMPORT_ERROR
    dh, H, G = SHAPES["dh128"]
    m = kv.Model(synth.preset("tiny", dtype="bf16", head_dim=dh, n_heads=H, n_kv_heads=G, n_layers=2),
                 None, seed=0, max_context=256, max_rows=64)
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    p = Pair(m, "dh128", "bf16", 5000).fill(1, 4900)
    seen = [4000, 4899]
    r = m.rows8([(p.c, seen)])
    big = Pair(m, "dh128", "bf16", 5000).fill(3, 5000)
    rb = m.rows8([(big.c, np.arange(4900, 5000))])
    q = queries(1, 2, p.H, p.dh, "bf16")
    qb = queries(2, 100, p.H, p.dh, "bf16")
    out, outb = torch.empty_like(q), torch.empty_like(qb)
    want = torch.empty_like(q)
    s = torch.cuda.Stream()
    m.set_stream(s.cuda_stream)
    try:
        torch.cuda.synchronize()
        r.attention(0, q, want, weigh=0.0)
        m.synchronize()
        with torch.cuda.stream(s):
            w = weights_of(p.c, 0, 4900, p.G)
        m.synchronize()
        k1 = torch.zeros((1, 2, p.G, p.dh), dtype=torch.bfloat16, device="cuda")
        kept = torch.zeros((2, p.G, 3), dtype=torch.int32, device="cuda")
        refused = []
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            r.attention(0, q, out, weigh=1.0)
            for call in (lambda: p.c.write([0], k1, k1), lambda: p.c.keep(kept),
                         lambda: r.move(seen), lambda: m.cache8(5),
                         lambda: m.rows8([(p.c, [1])]),
                         lambda: rb.attention(0, qb, outb, weigh=0.0)):
                try:
                    call()
                    refused.append(0)
                except kv.KvrError as e:
                    refused.append(e.code)
        assert refused == [6] * 6
        out.fill_(float("nan"))
        with torch.cuda.stream(s):
            g.replay()
            rb.attention(0, qb, outb, weigh=0.0)
            g.replay()
        m.synchronize()
        torch.cuda.synchronize()
    finally:
        m.set_stream(torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out, want)
    check_attention(big, 0, qb, np.arange(4900, 5000), outb, weights_of(big.c, 0, 5000, p.G))
    got = weights_of(p.c, 0, 4900, p.G)
    assert torch.allclose(got, 3 * w, rtol=2.0 ** -22, atol=0)  # two more sums of one rounding each
    m.close()


@pytest.mark.parametrize("rows_", [2, 200, 1500])
def test_captured_before_any_other_call(models, rows_):
    """Rows whose first call is captured, and calls that follow the upload of their tables at once."""
    m, n = models("dh128", "bf16"), 1600
    p = Pair(m, "dh128", "bf16", n).fill(31, n)
    seen = np.linspace(7, n - 1, rows_).astype(int)
    q = queries(32, rows_, p.H, p.dh, "bf16")
    first = m.rows8([(p.c, seen)])
    want, out, again = torch.empty_like(q), torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    s = torch.cuda.Stream()
    m.set_stream(s.cuda_stream)
    try:
        torch.cuda.synchronize()
        first.attention(0, q, want, weigh=0.0)  # (the scratch grows)
        r = m.rows8([(p.c, np.zeros(rows_, int))])
        m.synchronize()
        r.move(seen)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            r.attention(0, q, out, weigh=0.0)
        r.attention(0, q, again, weigh=0.0)
        m.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        m.synchronize()
        torch.cuda.synchronize()
    finally:
        m.set_stream(torch.cuda.current_stream().cuda_stream)
    assert torch.equal(again, want) and torch.equal(out, want)
    r.close()
    first.close()
    p.c.close()


def test_refused_capture_leaves_nothing():
    """A captured call whose scratch has not grown: nothing of it is in the graph, of the documents
    that come before the one that wants it either."""
    if kv is None:
        raise _IMPORT_ERROR
    dh, H, G = SHAPES["dh128"]
    m = kv.Model(synth.preset("tiny", dtype="bf16", head_dim=dh, n_heads=H, n_kv_heads=G, n_layers=2),
                 None, seed=0, max_context=256, max_rows=64)
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    few = Pair(m, "dh128", "bf16", 100).fill(5, 100)
    many = Pair(m, "dh128", "bf16", 2000).fill(7, 2000)
    # few rows' scratch, larger than the call below wants, and none for many rows of a document
    warm = m.rows8([(few.c, np.sort(np.arange(400) % 100))])
    qw = queries(8, 400, H, dh, "bf16")
    warm.attention(0, qw, torch.empty_like(qw), weigh=0.0)
    r = m.rows8([(few.c, [50]), (many.c, np.arange(1700, 2000))])
    q = queries(9, 301, H, dh, "bf16")
    out, mark = torch.full_like(q, 7.0), torch.zeros(8, device="cuda")
    for d in (few, many):
        d.c.set_weights(torch.full((2, G, d.c.n), 3.0, device="cuda"))
    s = torch.cuda.Stream()
    m.set_stream(s.cuda_stream)
    try:
        torch.cuda.synchronize()
        before = m.launches()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            mark += 1
            with pytest.raises(kv.KvrError) as e:
                r.attention(0, q, out, weigh=0.5)
        assert e.value.code == 6 and m.launches() == before
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        assert (mark == 1).all() and (out == 7).all()
        with torch.cuda.stream(s):
            for d in (few, many):
                assert (weights_of(d.c, 0, d.c.n, G) == 3).all()
        r.attention(0, q, out, weigh=0.5)  # once, as if the refused one had not been
        m.synchronize()
    finally:
        m.set_stream(torch.cuda.current_stream().cuda_stream)
    check_attention(few, 0, q[:1], [50], out[:1], weights_of(few.c, 0, 100, G), np.full((G, 100), 3.0),
                    0.5)
    check_attention(many, 0, q[1:], np.arange(1700, 2000), out[1:], weights_of(many.c, 0, 2000, G),
                    np.full((G, 2000), 3.0), 0.5)
    m.close()


def test_outgrown_scratch_is_freed():
    """Rows of a document, of more of it from call to call: a model that has captured nothing holds as
    much then as one that made the last call alone."""
    if kv is None:
        raise _IMPORT_ERROR
    dh, H, G, R, ends = 128, 16, 8, 1021, [2600, 5500, 11800, 25000, 53000]

    def grown(ends):
        m = kv.Model(synth.preset("tiny", dtype="bf16", head_dim=dh, n_heads=H, n_kv_heads=G,
                                  n_layers=1), None, seed=0, max_context=256, max_rows=64)
        m.set_stream(torch.cuda.current_stream().cuda_stream)
        c, at = m.cache8(ends[-1]), 10000
        for i in range(0, ends[-1], at):
            n = min(at, ends[-1] - i)
            k = torch.ones((n, 1, G, dh), dtype=torch.bfloat16, device="cuda")
            c.write(np.arange(i, i + n), k, k)
        r = m.rows8([(c, np.arange(R))])
        q = torch.ones((R, H, dh), dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        free = torch.cuda.mem_get_info()[0]
        for e in ends:
            r.move(np.arange(e - R, e))
            before = m.launches()
            r.attention(0, q, out, weigh=0.0)
            assert (out == 1).all()
        assert m.launches() - before >= 5  # by way of pages of halves: the most scratch
        torch.cuda.synchronize()
        used = free - torch.cuda.mem_get_info()[0]
        m.close()
        return used

    grown(ends)  # (all kernels are loaded)
    last, all_ = grown(ends[-1:]), grown(ends)
    assert last > 200e6
    assert all_ - last < 0.1 * last, (last, all_)


def test_refusals(models):
    m = models("dh64", "bf16")
    dh, H, G = SHAPES["dh64"]
    p = Pair(m, "dh64", "bf16", 100).fill(1, 50)
    one = torch.zeros((1, 2, G, dh), dtype=torch.bfloat16, device="cuda")
    lib, c = kv._lib, p.c

    def refused(code, f, *a, **kw):
        with pytest.raises(kv.KvrError) as e:
            f(*a, **kw)
        assert e.value.code == code, e.value

    refused(2, m.cache8, 0)
    refused(2, m.cache8, (1 << 20) + 1)
    refused(2, c.write, [51], one, one)       # a gap
    refused(2, c.write, [-1], one, one)
    refused(2, c.write, [100], one, one)
    refused(2, c.read, [50], one, one)
    two = torch.zeros((2, 2, G, dh), dtype=torch.bfloat16, device="cuda")
    refused(2, c.write, [5, 5], two, two)
    for call in (c.write, c.read):  # another type, host memory, another size: the binding's own
        with pytest.raises(ValueError):
            call([5], one.float(), one)
        with pytest.raises(ValueError):
            call([5], one.cpu(), one)
        with pytest.raises(ValueError):
            call([5], two, one)
    host = np.zeros(4096, np.int32)
    i5 = np.array([5], np.int32)
    assert lib.kvr_c8_write(c.h, i5.ctypes.data, 1, 0, 2, host.ctypes.data, host.ctypes.data) == 1
    assert lib.kvr_c8_write(c.h, i5.ctypes.data, 1, 0, 2, one.data_ptr() + 2, one.data_ptr()) == 1
    assert lib.kvr_c8_write(c.h, i5.ctypes.data, 1, 0, 3, one.data_ptr(), one.data_ptr()) == 2
    assert lib.kvr_c8_read(c.h, i5.ctypes.data, -1, 0, 2, one.data_ptr(), one.data_ptr()) == 2
    assert lib.kvr_c8_write(c.h, None, 1, 0, 2, one.data_ptr(), one.data_ptr()) == 1
    num = torch.zeros((2, G, 51), dtype=torch.int32, device="cuda")
    refused(2, c.entries, num)
    assert lib.kvr_c8_entries(c.h, 5, 0, 2, host.ctypes.data, None) == 1
    assert lib.kvr_c8_entries(c.h, 5, 0, 2, None, None) == 0
    assert lib.kvr_c8_set_weights(c.h, 5, 0, 2, None) == 1
    kept = torch.zeros((2, G, 20), dtype=torch.int32, device="cuda")
    refused(2, c.choose, torch.zeros((2, G, 51), dtype=torch.int32, device="cuda"))
    refused(2, c.choose, kept, first=11, recent=10)
    refused(2, c.choose, kept, first=-1)
    refused(2, c.choose, kept, recent=2 ** 31 - 1)
    refused(2, c.keep, kept, into=m.cache8(19))
    refused(2, c.keep, torch.zeros((2, G, 51), dtype=torch.int32, device="cuda"))
    other = models("dh64", "fp32")
    refused(1, c.keep, kept, into=other.cache8(50))
    refused(1, other.rows8, [(c, [1])])
    refused(1, m.rows8, [(c, [1]), (c, [2])])  # one document twice
    refused(2, m.rows8, [(c, [100])])
    refused(2, m.rows8, [(c, [-2])])
    refused(2, m.rows8, [(c, [5, 4])])
    refused(2, m.rows8, [(c, [])])
    r = m.rows8([(c, [60])])
    q = queries(1, 1, H, dh, "bf16")
    out = torch.empty_like(q)
    refused(2, r.attention, 0, q, out)  # not held yet
    r.move([49])
    refused(2, r.attention, 2, q, out)
    refused(2, r.attention, 0, q, out, weigh=1.5)
    refused(2, r.attention, 0, q, out, weigh=float("nan"))
    assert lib.kvr_c8_attention(r.h, 0, q.data_ptr(), H * dh - 8, out.data_ptr()) == 1
    assert lib.kvr_c8_attention(r.h, 0, host.ctypes.data, H * dh, out.data_ptr()) == 1
    assert lib.kvr_c8_attention(r.h, 0, q.data_ptr(), H * dh, None) == 1
    with pytest.raises(ValueError):
        r.move([1, 2])
    r.attention(0, q, out)
    p.check()  # nothing of the above changed it
    c.keep(kept[:, :, :1].contiguous() * 0)
    refused(2, r.attention, 0, q, out)  # the row lies past what is left
    r.move([0])
    r.attention(0, q, out)
    c.close()
    refused(1, r.attention, 0, q, out)
    refused(1, r.move, [0])
    r.close()
