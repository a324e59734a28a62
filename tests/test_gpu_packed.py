"""The packed cache against its plain 64-bit form (tests/packed_plain.py): stored values, bounds
and selections exactly, attention within the roundings of its types."""
import numpy as np
import pytest
import torch

from paper_2609_17983_gb300 import synth
from tests import packed_plain as pp

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


def read(doc, positions, layers, G, dh, dtype, **kw):
    k = torch.empty((len(positions), layers, G, dh), dtype=TORCH[dtype], device="cuda")
    v = torch.empty_like(k)
    doc.read(positions, k, v, **kw)
    return f64(k), f64(v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", ["dh64", "dh128"])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 200])
def test_store_and_bounds(models, shape, dtype, n):
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    k, v = rows(n, n, 2, G, dh, dtype), rows(n + 1, n, 2, G, dh, dtype)
    doc = m.packed(n + 5)
    doc.write(np.arange(n), k, v)
    assert doc.n == n
    want = pp.stored(f64(k)), pp.stored(f64(v))
    got = read(doc, np.arange(n), 2, G, dh, dtype)
    assert same(got[0], want[0]) and same(got[1], want[1])
    for l in range(2):
        hi, lo, u = doc.bounds(l)
        whi, wlo, wu = pp.bounds(want[0][:, l])
        assert same(u, wu) and same(hi, whi) and same(lo, wlo)
    # scattered positions of one layer, in place: the rest and the other layer stay
    at = np.unique(np.r_[0, n // 3, n // 2, n - 1])
    k2, v2 = rows(5, len(at), 1, G, dh, dtype), rows(6, len(at), 1, G, dh, dtype)
    doc.write(at, k2, v2, layer_begin=1)
    want[0][at, 1], want[1][at, 1] = pp.stored(f64(k2))[:, 0], pp.stored(f64(v2))[:, 0]
    got = read(doc, np.arange(n), 2, G, dh, dtype)
    assert same(got[0], want[0]) and same(got[1], want[1])
    for l in range(2):
        assert all(same(a, b) for a, b in zip(doc.bounds(l)[:2], pp.bounds(want[0][:, l])[:2]))
    got = read(doc, at, 1, G, dh, dtype, layer_begin=0, layer_end=1)
    assert same(got[0], want[0][at, :1]) and same(got[1], want[1][at, :1])
    # appended behind, two blocks at once where they end
    k3, v3 = rows(7, 5, 2, G, dh, dtype), rows(8, 5, 2, G, dh, dtype)
    doc.write(np.arange(n, n + 5), k3, v3)
    got = read(doc, np.arange(n - 1, n + 5), 2, G, dh, dtype)
    assert doc.n == n + 5 and same(got[0][1:], pp.stored(f64(k3)))
    assert same(got[1], np.r_[want[1][-1:], pp.stored(f64(v3))])
    doc.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_store_edges_of_the_grids(models, dtype):
    """Ties of codes and scales, zeros, the smallest and largest scales, NaN and infinity."""
    dh, H, G = SHAPES["dh64"]
    m = models("dh64", dtype)
    x = torch.zeros((64, 2, G, dh))
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for i in range(32):  # midpoints of the codes at 32 scales; signs mixed
        s = (8 + i % 8) / 8 * 2.0 ** (i // 8 * 7 - 14)
        x[i, :, :, :8], x[i, :, :, 8:16] = mid * s, -mid * s
        x[i, :, :, 16:24] = mid * s * (1 + 2.0 ** -7)
        x[i, :, :, 24] = 6 * s
        x[i, :, :, 32] = (16.5 + i % 8) / 16 * 6 * 2.0 ** (i - 20)  # halfway between scales
        x[i, :, :, 48] = 6 * 2.0 ** -18 * (1 + i)  # multiples of half the least scale
    x[32, :, :, 0], x[33, 0, 0, 63], x[34, 1, 1, 5], x[35, :, 1, 0] = 3e38, float("nan"), float(
        "inf"), -float("inf")
    x[36] = 1e-30
    x[37] = 61440.0
    x[38, :, :, 3] = 65504.0
    x = x.to(TORCH[dtype])
    doc = m.packed(64)
    doc.write(np.arange(64), x.cuda(), x.flip(0).contiguous().cuda())
    got = read(doc, np.arange(64), 2, G, dh, dtype)
    assert same(got[0], pp.stored(f64(x))) and same(got[1], pp.stored(f64(x.flip(0))))
    for l in range(2):
        assert all(same(a, b) for a, b in zip(doc.bounds(l), pp.bounds(pp.stored(f64(x))[:, l])))
    doc.close()


@pytest.mark.parametrize("shape,dtype,pages,most", [
    ("dh128", "bf16", 300, 6), ("dh64", "bf16", 420, 3), ("dh64", "fp32", 400, 3)])
def test_store_some_rows_of_pages(models, shape, dtype, pages, most):
    """A few rows of each of more blocks than the chip takes at once, then many rows of three
    pages: next to one another or not, with a NaN and an infinity among them."""
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    n = 64 * pages - 7
    k, v = rows(1, n, 2, G, dh, dtype), rows(2, n, 2, G, dh, dtype)
    doc = m.packed(n)
    doc.write(np.arange(n), k, v)
    rng = np.random.default_rng(pages)
    few = [64 * p + rng.permutation(57)[:rng.integers(0 if p else most, most + 1)]
           for p in range(pages)]
    many = [64 * p + rng.permutation(57)[:41] for p in (0, 5, pages - 1)]
    for at in (few, many):
        at = np.sort(np.concatenate(at))
        k2, v2 = rows(3, len(at), 2, G, dh, dtype), rows(4, len(at), 2, G, dh, dtype)
        k2[len(at) // 2, 1, G - 1, 3], v2[len(at) // 3, 0, 0, dh - 1] = float("nan"), float("inf")
        doc.write(at, k2, v2)
        where = torch.from_numpy(at).cuda()
        k[where], v[where] = k2, v2
    want = pp.stored(f64(k)), pp.stored(f64(v))
    got = read(doc, np.arange(n), 2, G, dh, dtype)
    assert same(got[0], want[0]) and same(got[1], want[1])
    for l in range(2):
        assert all(same(a, b) for a, b in zip(doc.bounds(l), pp.bounds(want[0][:, l])))
    doc.close()


def test_store_many_scattered_rows(models):
    """More scattered positions than come with a launch."""
    dh, H, G = SHAPES["dh64"]
    m = models("dh64", "bf16")
    n = 2000
    k, v = rows(1, n, 2, G, dh, "bf16"), rows(2, n, 2, G, dh, "bf16")
    doc = m.packed(n)
    doc.write(np.arange(n), k, v)
    at = np.sort(np.random.default_rng(0).permutation(n)[:700])
    k2, v2 = rows(3, 700, 2, G, dh, "bf16"), rows(4, 700, 2, G, dh, "bf16")
    doc.write(at, k2, v2)
    want = pp.stored(f64(k)), pp.stored(f64(v))
    want[0][at], want[1][at] = pp.stored(f64(k2)), pp.stored(f64(v2))
    got = read(doc, np.arange(n), 2, G, dh, "bf16")
    assert same(got[0], want[0]) and same(got[1], want[1])
    got = read(doc, at, 2, G, dh, "bf16")
    assert same(got[0], want[0][at]) and same(got[1], want[1][at])
    doc.close()


def bound(dtype, ref, vmax, smax):
    """What the roundings allow.  bf16: the output to 8 bits (off by at most 2^-8 of itself), the
    weights to 11 (so at most 2^-11 of the largest value), the scores' and exponentials'
    fp32.  fp32: weights to 22 bits; a score is a sum of 8 (head size 128) products of fragments in two parts,
    each addition off by at most 2^-23 of the sum of magnitudes, and its error
    moves a weight by as much, relatively, and the result by at most twice
    that of the largest value."""
    delta = 2.0 ** -19 + 16 * 2.0 ** -23 * smax
    if dtype == "bf16":
        return (2.0 ** -8 * np.abs(ref) +
                (2.0 ** -11 + 2 * delta)[..., None] * vmax[..., None])
    return (2 * delta * vmax)[..., None] + 2.0 ** -24 * np.abs(ref)


def check(got, q, pos, k, v, dtype, blocks=None):
    ref, vmax, smax = pp.attention(q, pos, k, v, blocks)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    err = np.abs(got - ref) - bound(dtype, ref, vmax, smax)
    assert not (err > 0).any(), float(np.nanmax(err))


def queries(seed, R, H, dh, dtype, size=1.5):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn((R, H, dh), generator=g)).to(TORCH[dtype]).cuda()


def document(m, seed, n, shape, dtype, capacity=None):
    dh, H, G = SHAPES[shape]
    doc = m.packed(capacity or max(n, 1))
    k, v = rows(seed, n, 2, G, dh, dtype), rows(seed + 1, n, 2, G, dh, dtype)
    if n:
        doc.write(np.arange(n), k, v)
    return doc, pp.stored(f64(k)), pp.stored(f64(v))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("n,R", [(1, 1), (64, 1), (65, 3), (500, 1), (1000, 13)])
def test_attention_one_document(models, shape, dtype, n, R):
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    doc, k, v = document(m, n, n, shape, dtype, n + 70)
    pos = np.sort(np.random.default_rng(n).integers(-1, n, R))
    pos[-1] = n - 1
    r = m.rows([(doc, pos)])
    q = queries(n + R, R, H, dh, dtype)
    out = torch.full_like(q, float("nan"))
    r.attention(1, q, out)
    check(f64(out), f64(q), pos, k[:, 1], v[:, 1], dtype)
    r.close()
    doc.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_several_documents_and_moves(models, dtype):
    dh, H, G = SHAPES["dh128"]
    m = models("dh128", dtype)
    lens = [0, 1, 300, 129, 64]
    docs = [document(m, 10 * i + 3, n, "dh128", dtype, n + 3) for i, n in enumerate(lens)]
    pos = [[-1], [-1, 0], [5, 5, 299], [], [0, 63]]
    r = m.rows([(d[0], p) for d, p in zip(docs, pos)])
    q = queries(1, r.n, H, dh, dtype)
    for move in range(2):
        if move:
            pos = [[-1], [0, 0], [0, 130, 131], [], [-1, -1]]
            r.move(np.concatenate(pos).astype(np.int32))
        out = torch.full_like(q, float("nan"))
        r.attention(0, q, out)
        i = 0
        for (doc, k, v), p in zip(docs, pos):
            if p:
                check(f64(out[i:i + len(p)]), f64(q[i:i + len(p)]), np.array(p), k[:, 0], v[:, 0],
                      dtype)
            i += len(p)
    r.close()


@pytest.mark.parametrize("shape,n,R,spread", [("dh64", 4000, 1201, True), ("dh128", 2000, 300, False),
                                              ("dh128", 2049, 501, True)])
def test_attention_many_rows(models, shape, n, R, spread):
    """Rows that go by way of unpacked pages: odd
    lengths, rows that see nothing, a second document with few rows, q rows apart, NaN."""
    dh, H, G = SHAPES[shape]
    m = models(shape, "bf16")
    k, v = rows(n, n, 2, G, dh, "bf16"), rows(n + 1, n, 2, G, dh, "bf16")
    k[n - 10, :, 0, 7], v[n - 5, :, G - 1, 3] = float("nan"), float("inf")
    doc = m.packed(n + 1)
    doc.write(np.arange(n), k, v)
    k, v = pp.stored(f64(k)), pp.stored(f64(v))
    small, ks, vs = document(m, 5, 100, shape, "bf16")
    pos = np.linspace(0, n - 1, R).astype(int) if spread else np.arange(n - R, n)
    pos[:3] = -1
    r = m.rows([(small, [50]), (doc, pos)])
    wide = torch.randn((R + 1, H + 2 * G, dh), device="cuda").bfloat16()
    q = wide[:, :H]
    out = torch.full((R + 1, H, dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    before = m.launches()
    r.attention(1, q, out)
    assert m.launches() - before >= 3  # the small document's, the unpacking, the attention
    check(f64(out[:1]), f64(q[:1]), np.array([50]), ks[:, 1], vs[:, 1], "bf16")
    check(f64(out[1:]), f64(q[1:]), pos, k[:, 1], v[:, 1], "bf16")
    assert (out[1:4] == 0).all()
    again = torch.empty_like(out)
    r.attention(1, q.contiguous(), again)
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(again))
    # the block lists of such rows are the fused kernel's
    blocks = torch.empty((R + 1, G, 3), dtype=torch.int32, device="cuda")
    r.select(1, q, blocks)
    r.attention(1, q, again, blocks=blocks)
    some = np.r_[1, 5, R - 20, R]  # row 1: a row that sees nothing
    b = blocks.cpu().numpy()[some]
    assert np.array_equal(b, pp.select(f64(q[some]), pos[some - 1], k[:, 1], 3))
    check(f64(again[some]), f64(q[some]), pos[some - 1], k[:, 1], v[:, 1], "bf16", b)
    r.close()
    doc.close()


def test_attention_rows_apart_sizes_and_streams(models):
    """q as a slice of wider rows; queries of very different sizes; a stream of its own."""
    dh, H, G = SHAPES["dh128"]
    m = models("dh128", "bf16")
    doc, k, v = document(m, 3, 400, "dh128", "bf16")
    pos = np.array([10, 200, 399])
    r = m.rows([(doc, pos)])
    wide = torch.randn((3, H + 2 * G, dh), device="cuda").bfloat16()
    wide[0] *= 1e-6
    wide[2] *= 4.0
    wide[1, 0, 5:] *= 2.0 ** -30  # entries of one vector far apart
    q = wide[:, :H]
    out = torch.empty((3, H, dh), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    m.set_stream(s.cuda_stream)
    r.attention(1, q, out)
    m.synchronize()
    m.set_stream(torch.cuda.current_stream().cuda_stream)
    check(f64(out), f64(q), pos, k[:, 1], v[:, 1], "bf16")
    again = torch.empty_like(out)
    r.attention(1, q.contiguous(), again)
    assert torch.equal(out, again)
    r.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_not_finite(models, dtype):
    """A NaN or infinity in a stored row, or in a query, reaches the rows that see it alone."""
    dh, H, G = SHAPES["dh128"]
    m = models("dh128", dtype)
    n = 200
    k, v = rows(1, n, 2, G, dh, dtype), rows(2, n, 2, G, dh, dtype)
    k[100, :, 0, 7] = float("nan")
    v[130, :, 1, 3] = float("inf")
    doc = m.packed(n)
    doc.write(np.arange(n), k, v)
    pos = np.array([50, 99, 100, 129, 130, 199])
    r = m.rows([(doc, pos)])
    q = queries(4, len(pos), H, dh, dtype)
    out = torch.empty_like(q)
    r.attention(0, q, out)
    ks, vs = pp.stored(f64(k))[:, 0], pp.stored(f64(v))[:, 0]
    check(f64(out), f64(q), pos, ks, vs, dtype)
    got = f64(out).reshape(len(pos), G, -1)
    assert np.isnan(got).all(2).tolist() == [[False, False], [False, False], [True, False],
                                             [True, False], [True, True], [True, True]]
    q[1, 3, 5] = float("nan")  # the heads of that row's KV head alone
    r.attention(0, q, out)
    bad = np.isnan(f64(out)).any(2)
    assert bad[1].tolist() == [h == 3 for h in range(H)] and not bad[0].any()
    r.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("n,count", [(1, 1), (64, 2), (700, 1), (700, 4), (700, 11), (700, 40)])
def test_selection_and_block_attention(models, shape, dtype, n, count):
    dh, H, G = SHAPES[shape]
    m = models(shape, dtype)
    doc, k, v = document(m, n + count, n, shape, dtype)
    pos = np.sort(np.random.default_rng(count).integers(-1, n, 5))
    pos[-1] = n - 1
    r = m.rows([(doc, pos)])
    q = queries(n, 5, H, dh, dtype)
    blocks = torch.full((5, G, count), 7777, dtype=torch.int32, device="cuda")
    r.select(1, q, blocks)
    want = pp.select(f64(q), pos, k[:, 1], count)
    assert np.array_equal(blocks.cpu().numpy(), want)
    out = torch.full_like(q, float("nan"))
    r.attention(1, q, out, blocks=blocks)
    check(f64(out), f64(q), pos, k[:, 1], v[:, 1], dtype, want)
    r.close()


def test_selection_ties_and_queries_that_are_not_finite(models):
    dh, H, G = SHAPES["dh64"]
    m = models("dh64", "bf16")
    n = 1000
    doc = m.packed(n)
    one = rows(1, 1, 2, G, dh, "bf16").expand(n, 2, G, dh).contiguous()  # blocks all alike
    doc.write(np.arange(n), one, one)
    r = m.rows([(doc, [999, 999, 999])])
    q = queries(2, 3, H, dh, "bf16")
    q[1, 0, 0], q[2] = float("inf"), 0.0
    blocks = torch.empty((3, G, 6), dtype=torch.int32, device="cuda")
    r.select(0, q, blocks)
    assert blocks.cpu().tolist() == [[[0, 1, 2, 3, 4, 15]] * G] * 3
    r.close()


@pytest.mark.parametrize("n", [3000, 20000])
def test_selection_of_scores_far_apart(models, n):
    """Scores of both signs over 30 binades, many of them equal, zeros among them."""
    dh, H, G = SHAPES["dh64"]
    m = models("dh64", "bf16")
    rng = np.random.default_rng(n)
    blocks = -(-n // 64)
    factor = np.sign(rng.normal(size=blocks)) * np.exp2(rng.integers(-18, 12, blocks))
    factor[rng.integers(0, blocks, blocks // 4)] = 0.0
    one = rows(3, 64, 1, G, dh, "bf16")
    x = torch.cat([one * float(f) for f in factor])[:n].expand(n, 2, G, dh).contiguous()
    doc = m.packed(n)
    doc.write(np.arange(n), x, x)
    pos = [n // 2, n - 1]
    r = m.rows([(doc, pos)])
    q = queries(4, 2, H, dh, "bf16")
    k = read(doc, np.arange(n), 2, G, dh, "bf16")[0][:, 0]
    for count in (1, 2, 7, blocks // 3, blocks - 2):
        got = torch.empty((2, G, count), dtype=torch.int32, device="cuda")
        r.select(0, q, got)
        assert np.array_equal(got.cpu().numpy(), pp.select(f64(q), np.array(pos), k, count))
    r.close()


def test_block_lists_of_the_caller(models):
    """Any order, entries outside the row's reach, none at all, long lists."""
    dh, H, G = SHAPES["dh128"]
    m = models("dh128", "bf16")
    doc, k, v = document(m, 9, 1000, "dh128", "bf16")
    pos = np.array([-1, 130, 700, 999])
    r = m.rows([(doc, pos)])
    q = queries(3, 4, H, dh, "bf16")
    lists = np.full((4, G, 300), -1, np.int32)
    lists[0, :, :3] = [0, 1, 2]
    lists[1, 0, :5] = [2, 0, 3, -5, 2 ** 31 - 1]  # of which the row sees 2 and 0
    lists[2, 0, 299] = 4  # the last of a long list; the other KV head has none
    lists[3, :, ::20] = np.arange(15)[::-1]
    out = torch.empty_like(q)
    r.attention(1, q, out, blocks=torch.from_numpy(lists).cuda())
    got = f64(out)
    check(got, f64(q), pos, k[:, 1], v[:, 1], "bf16", lists.astype(np.int64))
    assert (got[0] == 0).all() and (got[2, H // G:] == 0).all()
    r.close()


def test_long_cache_offsets(models):
    """A cache whose blocks lie past 2^32 bytes: its last layer's rows."""
    dh, H, G = SHAPES["dh128"]
    m = models("dh128", "bf16", 40)
    n = 1 << 20
    doc = m.packed(n)  # 40 layers x 2 heads x 2^14 blocks x 9216 bytes = 12 GB
    k, v = rows(1, 300, 1, G, dh, "bf16"), rows(2, 300, 1, G, dh, "bf16")
    doc.write(np.arange(300), k, v, layer_begin=39)
    # the far end: zeros in between
    step = 1 << 17
    z = torch.zeros((step, 1, G, dh), dtype=torch.bfloat16, device="cuda")
    for p in range(300, n, step):
        c = min(step, n - p)
        doc.write(np.arange(p, p + c), z[:c], z[:c], layer_begin=39)
    doc.write(np.arange(n - 300, n), k, v, layer_begin=39)
    got = read(doc, np.arange(n - 300, n), 1, G, dh, "bf16", layer_begin=39)
    ks, vs = pp.stored(f64(k)), pp.stored(f64(v))
    assert same(got[0], ks) and same(got[1], vs)
    r = m.rows([(doc, [n - 1])])
    q = queries(5, 1, H, dh, "bf16")
    blocks = torch.tensor([[[0, 1, n // 64 - 2, n // 64 - 1]] * G], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    r.attention(39, q, out, blocks=blocks)
    kk, vv = np.zeros((512, G, dh)), np.zeros((512, G, dh))  # four blocks; those three rows' ends
    kk[:128], vv[:128] = ks[:128, 0], vs[:128, 0]
    kk[128:256], vv[128:256] = ks[-128:, 0], vs[-128:, 0]
    check(f64(out), f64(q), np.array([255]), kk, vv, "bf16")
    chosen = torch.empty((1, G, 9), dtype=torch.int32, device="cuda")
    r.select(39, q, chosen)
    at = sorted(set(range(5)) | set(range(n // 64 - 5, n // 64)))  # the blocks that are not zero
    assert set(chosen.cpu().numpy().reshape(-1).tolist()) <= set(range(6)) | set(at)
    dense = torch.empty_like(q)
    r.attention(39, q, dense)
    assert torch.isfinite(dense).all()
    r.close()
    doc.close()


def test_refusals(models):
    dh, H, G = SHAPES["dh64"]
    m = models("dh64", "bf16")
    other = models("dh64", "fp32")
    k = rows(1, 4, 2, G, dh, "bf16")

    def code(f):
        with pytest.raises(kv.KvrError) as e:
            f()
        return e.value.code
    assert code(lambda: m.packed(0)) == 2 and code(lambda: m.packed((1 << 20) + 1)) == 2
    doc = m.packed(10)
    p = k.data_ptr()
    w = lambda at, l0=0, l1=2, kp=p, vp=p: kv.kvr_packed_write(doc.h, at, l0, l1, kp, vp)  # noqa: E731
    assert code(lambda: w([1])) == 2 and code(lambda: w([0, 2])) == 2  # gaps
    assert code(lambda: w([0, 0])) == 2 and code(lambda: w([1, 0])) == 2
    assert code(lambda: w([-1])) == 2 and code(lambda: w([0], -1, 2)) == 2
    assert code(lambda: w([0], 0, 3)) == 2 and code(lambda: w([0], 2, 1)) == 2
    assert code(lambda: w([0], kp=None)) == 1 and code(lambda: w([0], vp=p + 2)) == 1
    host = np.zeros(4 * 2 * G * dh + 8, np.uint16)
    at16 = host.ctypes.data + (-host.ctypes.data) % 16
    assert code(lambda: w([0], kp=at16)) == 1
    assert doc.n == 0
    w([])  # nothing
    w([0], 1, 1)
    assert doc.n == 0
    doc.write(np.arange(4), k, k)
    assert code(lambda: doc.read([4], k[:1], k[:1])) == 2
    with pytest.raises(ValueError):
        doc.write(np.arange(4), k.float(), k.float())
    with pytest.raises(ValueError):
        doc.write(np.arange(3), k, k)
    with pytest.raises(ValueError):
        doc.write(np.arange(4), k.cpu(), k.cpu())
    assert code(lambda: m.rows([(doc, [4])])) == 2 and code(lambda: m.rows([(doc, [-2])])) == 2
    assert code(lambda: m.rows([(doc, [2, 1])])) == 2 and code(lambda: m.rows([(doc, [])])) == 2
    assert code(lambda: other.rows([(doc, [0])])) == 1 and code(lambda: m.rows([])) == 2
    r = m.rows([(doc, [3])])
    q = queries(1, 1, H, dh, "bf16")
    out = torch.empty_like(q)
    assert code(lambda: r.attention(2, q, out)) == 2 and code(lambda: r.attention(-1, q, out)) == 2
    assert code(lambda: kv.kvr_packed_attention(r.h, 0, q.data_ptr(), H * dh - 8, out.data_ptr())) == 1
    assert code(lambda: kv.kvr_packed_attention(r.h, 0, q.data_ptr(), H * dh + 1, out.data_ptr())) == 1
    assert code(lambda: kv.kvr_packed_attention(r.h, 0, None, H * dh, out.data_ptr())) == 1
    assert code(lambda: kv.kvr_packed_attention(r.h, 0, at16, H * dh, out.data_ptr())) == 1
    assert code(lambda: kv.kvr_packed_select(r.h, 0, q.data_ptr(), H * dh, 0, out.data_ptr())) == 2
    assert code(lambda: kv.kvr_packed_attention_blocks(r.h, 0, q.data_ptr(), H * dh, out.data_ptr(),
                                                       16385, out.data_ptr())) == 2
    with pytest.raises(ValueError):
        r.attention(0, q.float(), out)
    with pytest.raises(ValueError):
        r.move([1, 2])
    assert code(lambda: r.move([9])) == 2
    r.attention(0, q, out)  # as before
    check(f64(out), f64(q), np.array([3]), pp.stored(f64(k))[:, 0], pp.stored(f64(k))[:, 0], "bf16")
    doc.close()
    assert code(lambda: r.attention(0, q, out)) == 1 and code(lambda: r.move([1])) == 1
    r.close()


def test_no_allocation_once_it_fits(models):
    dh, H, G = SHAPES["dh128"]
    m = models("dh128", "bf16")
    doc, k, v = document(m, 1, 600, "dh128", "bf16")
    r = m.rows([(doc, [599])])
    q = queries(1, 1, H, dh, "bf16")
    out, blocks = torch.empty_like(q), torch.empty((1, G, 4), dtype=torch.int32, device="cuda")

    def step():
        kk = rows(1, 1, 2, G, dh, "bf16")
        doc.write([599], kk, kk)
        r.select(0, q, blocks)
        r.attention(0, q, out, blocks=blocks)
        r.attention(0, q, out)
        m.synchronize()
    step()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        step()
    assert torch.cuda.mem_get_info()[0] == free
    r.close()
