"""Many rows of a document over an 8-bit cache, by each way that its kernels take (heads of 64 and
128, tiles whose pages are split and whole ones, weights in one run and several): the way is read
from the kernels that a call launches, its results are compared with 64 bits on the GPU."""
import numpy as np
import pytest
import torch

from paper_2609_17983_gb300 import synth
from tests.test_gpu_c8 import out_bound, score_error

try:
    from paper_2609_17983_gb300 import kvrepair as kv
except ImportError as _e:  # pragma: no cover
    kv, _IMPORT_ERROR = None, _e

pytestmark = pytest.mark.gpu

# way, whether a tile's pages are split, head size, heads, KV heads, entries up to the last row's, rows,
# spread over all entries or the last ones
CASES = {
    "straight_64": ("straight", True, 64, 16, 2, 2999, 301, False),
    "straight_64_spread": ("straight", True, 64, 16, 2, 12343, 301, True),
    "straight_64_whole": ("straight", False, 64, 16, 2, 2001, 1021, True),
    "straight_64_tiny_heads": ("straight", True, 64, 4, 2, 12345, 511, False),
    "pages_64": ("pages", True, 64, 16, 2, 5003, 509, True),
    "pages_64_runs": ("pages", True, 64, 16, 2, 3001, 701, False),
    "pages_64_whole": ("pages", False, 64, 16, 2, 3001, 2049, False),
    "straight_128": ("straight", True, 128, 14, 2, 3001, 301, True),
    "straight_128_whole": ("straight", False, 128, 14, 2, 2999, 1021, True),
    "straight_128_whole_one_run": ("straight", False, 128, 28, 4, 2001, 513, False),
    "pages_128": ("pages", True, 128, 14, 2, 3001, 509, True),
    "pages_128_runs": ("pages", True, 128, 14, 2, 3001, 701, False),
    "pages_128_whole": ("pages", False, 128, 16, 2, 3001, 2049, False),
    "fused_64": ("fused", True, 64, 16, 2, 700, 40, True),
    "fused_64_301": ("fused", True, 64, 16, 2, 5003, 301, True),
    "fused_64_509": ("fused", True, 64, 16, 2, 3001, 509, True),
    "fused_128": ("fused", True, 128, 14, 2, 700, 40, True),
}
BEHIND = 103  # entries past the last row's


@pytest.fixture(scope="module")
def models():
    if kv is None:
        raise _IMPORT_ERROR
    made = {}

    def get(dh, H, G):
        if (dh, H, G) not in made:
            m = kv.Model(synth.preset("tiny", dtype="bf16", head_dim=dh, n_heads=H, n_kv_heads=G,
                                      n_layers=1), None, seed=0, max_context=256, max_rows=64)
            m.set_stream(torch.cuda.current_stream().cuda_stream)
            made[dh, H, G] = m
        return made[dh, H, G]
    yield get
    for m in made.values():
        m.close()


def normal(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").bfloat16()


def filled(m, k, v):
    c = m.cache8(len(k))
    c.write(np.arange(len(k)), k[:, None], v[:, None])
    return c


def stored(c, n, G, dh):
    k, v = (torch.empty((n, 1, G, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.read(np.arange(n), k, v)
    return k[:, 0].double(), v[:, 0].double()


def weights(c, n, G):
    w = torch.full((1, G, n), 77.0, device="cuda")
    c.entries(None, w)
    return w[0].double()


def places(n, R, spread):
    return np.linspace(0, n - 1, R).astype(int) if spread else np.arange(n - R, n)


class Call:
    """A document with rows of a case, of which the first three see nothing, and one row of a short
    document; both ways of the call, their launches and their results."""

    def __init__(self, m, case, k, v, q, old=None, decay=0.0):
        way, split, dh, H, G, n, R, spread = CASES[case]
        self.seen = places(n, R, spread)
        self.seen[:3] = -1
        self.n, self.G, self.grp, self.q = len(k), G, H // G, q
        small = filled(m, normal(91, 70, G, dh), normal(92, 70, G, dh))
        c = filled(m, k, v)
        r = m.rows8([(small, [50]), (c, self.seen)])
        alone, self.out = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
        a = m.launches()
        r.attention(0, q, alone)
        b = m.launches()
        if old is not None:
            c.set_weights(old[None])
        e = m.launches()
        r.attention(0, q, self.out, weigh=decay)
        plain, weighing = b - a, m.launches() - e
        # one launch is the fused kernel's, for the rows that see nothing and the short document
        runs = -(-(-(-(R - 3) * self.grp // 128)) // 32)
        want = {"fused": (1, 2), "straight": (2 + split, 4 + split + (runs > 1)),
                "pages": (3 + split, 6 + split + (runs > 1))}[way]
        assert (plain, weighing) == want
        assert torch.equal(alone.view(torch.int16), self.out.view(torch.int16))
        self.k, self.v = stored(c, self.n, G, dh)
        self.weight = weights(c, self.n, G)
        self.small = [stored(small, 70, G, dh), weights(small, 70, G)]
        self.old = None if old is None or not decay else old.double() * decay
        r.close()
        c.close()
        small.close()

    def check(self, key_error=0.0, value_error=0.0):
        """key_error, value_error: how far a key's or value's entries may be from the stored ones."""
        self._document(self.q[:1], self.out[:1], np.array([50]), *self.small[0], self.small[1], None)
        self._document(self.q[1:], self.out[1:], self.seen, self.k, self.v, self.weight, self.old,
                       key_error, value_error)
        assert (self.out[1:4] == 0).all()

    def _document(self, q, out, seen, k, v, weight, old, key_error=0.0, value_error=0.0):
        n, dh, grp = len(k), k.shape[-1], self.grp
        last = torch.as_tensor(seen, device="cuda").repeat_interleave(grp)
        masked = torch.arange(n, device="cuda")[None] > last[:, None]
        for g in range(self.G):
            qg = q[:, g * grp:(g + 1) * grp].reshape(-1, dh).double()
            got = out[:, g * grp:(g + 1) * grp].reshape(-1, dh).double()
            x = (qg @ k[:, g].T / dh ** 0.5).masked_fill(masked, -float("inf"))
            x[~torch.isfinite(qg).all(1)] = float("nan")
            w = torch.softmax(x, -1)
            w[last < 0] = 0.0
            vz = torch.nan_to_num(v[:, g])  # who sees a marked entry is NaN by its key
            ref = w @ vz
            most = vz.abs().amax(1).cummax(0).values[last.clamp(min=0)]
            q1 = torch.nan_to_num(qg).abs()
            size = (q1 @ torch.nan_to_num(k[:, g]).abs().T / dh ** 0.5).masked_fill(masked, 0.0).amax(1)
            assert torch.equal(torch.isnan(got), torch.isnan(ref))
            # of a sum of exponentials: 20 additions in a step, one a step, in fp32
            sums = (n / 64 + 20) * 2.0 ** -24
            # a key's entries each off by key_error move its score by this, its weight and the sum of
            # all by as much
            moved = torch.expm1(2 * key_error * q1.sum(1) / dh ** 0.5)
            lim = torch.as_tensor(out_bound("bf16", ref.cpu().numpy(), most.cpu().numpy(),
                                            size.cpu().numpy()), device="cuda")
            lim += ((2 * sums + moved) * most)[:, None] + value_error
            err = (got - ref).abs() - lim
            assert not (err > 0).any(), (g, float(torch.nan_to_num(err, -1.0).max()))
            ok = torch.isfinite(w).all(1) & (last >= 0)
            total = w[ok].sum(0)
            part = (w[ok] * (3 * score_error(size) + sums + moved)[ok][:, None]).sum(0)
            was = torch.zeros_like(total) if old is None else old[g]
            lim = part + (len(qg) + 2) * 2.0 ** -24 * (total + was.abs()) + 2.0 ** -120
            err = (weight[g] - (was + total)).abs() - lim
            assert not (err > 0).any(), (g, float(err.max()))


@pytest.mark.parametrize("case", list(CASES))
def test_each_way(models, case):
    """Ragged sizes, marked entries, queries that are not finite, old weights that decay, and entries
    that no row sees, whose weights do."""
    way, split, dh, H, G, n, R, spread = CASES[case]
    m = models(dh, H, G)
    k, v = normal(1, n + BEHIND, G, dh), normal(2, n + BEHIND, G, dh)
    k *= torch.exp(0.7 * normal(3, G, dh).float()).bfloat16()
    k[n - 30, 0, 5], v[n - 20, G - 1, 7], k[n + 2] = float("nan"), float("inf"), float("nan")
    q = normal(4, R + 1, H, dh) * 1.5
    q[R // 2, 1, 3], q[R // 3, H - 1, 0] = float("nan"), float("inf")
    old = torch.rand((G, n + BEHIND), generator=torch.Generator().manual_seed(5)).cuda()
    Call(m, case, k, v, q, old, 0.5).check()
    old[:] = float("nan")
    Call(m, case, k, v, q, old, 0.0).check()  # a factor of zero forgets even that


@pytest.mark.parametrize("case", [c for c in CASES if "fused" not in c])
@pytest.mark.parametrize("size", [0.0, 2.0 ** -120])
def test_vanishing_products(models, case, size):
    """Keys of zero or tiny ones, queries of zero or tiny ones: equal weights for what a row sees."""
    way, split, dh, H, G, n, R, spread = CASES[case]
    m = models(dh, H, G)
    k = torch.full((n + BEHIND, G, dh), size, dtype=torch.bfloat16, device="cuda")
    q = normal(6, R + 1, H, dh)
    q[::2] = 0.0
    q[1::2] *= 2.0 ** -110
    Call(m, case, k, normal(7, n + BEHIND, G, dh), q).check()


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("keys,values", [(24, 24), (31, 31), (33, 33), (None, 40), (33, 40)])
def test_blocks_far_below_the_largest(models, case, keys, values):
    """A key and a value 2^keys and 2^values above the other blocks': those keep what lies above
    2^-32 of the largest power, in the output and in the weights; few rows keep all."""
    way, split, dh, H, G, n, R, spread = CASES[case]
    m = models(dh, H, G)
    g = torch.Generator(device="cuda").manual_seed(8)
    # scores of the same sign in all rows, so that weights of entries differ in their sums too
    u = torch.sign(torch.randn((G, dh), generator=g, device="cuda"))
    u[:, 0] = 0.0
    a = 0.25 + 1.25 * torch.rand((n + BEHIND, 1, 1), generator=g, device="cuda")
    k = (a * u).bfloat16()
    v = (1.5 + 0.25 * torch.rand((n + BEHIND, G, dh), generator=g, device="cuda")).bfloat16()
    q = 0.3 * u.repeat_interleave(H // G, 0)[None] + 0.05 * normal(9, R + 1, H, dh).float()
    q[:, :, 0] = 0.0  # the large key's only entry takes no part
    # codes of 1.5 to 1.75 under 2^-8 are 384 to 448
    key_power = value_power = 0.0
    if keys:
        key_power = 2.0 ** (keys - 8)
        k[100, :, 0] = 448 * key_power
    value_power = 2.0 ** (values - 8)
    v[n - 1, :, 0] = 448 * value_power  # seen by the last row alone
    call = Call(m, case, k, v, q.bfloat16())
    assert float(call.v[:n - 1 - n % 64].min()) >= 1.5 and float(call.v.max()) == 448 * value_power
    if way == "fused":
        call.check()
    else:
        call.check(2.0 ** -32 * key_power, 2.0 ** -32 * value_power)


@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("decay", [0.5, 1.0])
def test_entries_far_behind_the_last_row(models, case, decay):
    """Whole tiles of keys, and several CTAs' runs of them, that no row sees: their weights decay."""
    way, split, dh, H, G, n, R, spread = CASES[case]
    m, behind = models(dh, H, G), 4099
    k, v = normal(11, n + behind, G, dh), normal(12, n + behind, G, dh)
    old = torch.rand((G, n + behind), generator=torch.Generator().manual_seed(13)).cuda()
    call = Call(m, case, k, v, normal(14, R + 1, H, dh), old, decay)
    call.check()
    assert torch.equal(call.weight[:, n:], (old[:, n:] * decay).double())


@pytest.mark.parametrize("case", list(CASES))
def test_captured_and_replayed(models, case):
    """The first call of rows that have just been moved, captured: a replay is the call."""
    way, split, dh, H, G, n, R, spread = CASES[case]
    m = models(dh, H, G)
    c = filled(m, normal(15, n, G, dh), normal(16, n, G, dh))
    seen, q = places(n, R, spread), normal(17, R, H, dh)
    want, out = torch.empty_like(q), torch.full_like(q, 7.0)
    s = torch.cuda.Stream()
    try:
        torch.cuda.synchronize()
        m.set_stream(s.cuda_stream)
        first = m.rows8([(c, seen)])
        first.attention(0, q, want, weigh=0.0)  # (the scratch grows)
        first.attention(0, q, want, weigh=1.0)
        with torch.cuda.stream(s):
            twice = weights(c, n, G)
        r = m.rows8([(c, np.zeros(R, int))])
        m.synchronize()
        r.move(seen)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            r.attention(0, q, out, weigh=0.0)
            r.attention(0, q, out, weigh=1.0)
        with torch.cuda.stream(s):
            g.replay()
            g.replay()
        m.synchronize()
        torch.cuda.synchronize()
    finally:
        m.set_stream(torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out, want) and torch.equal(weights(c, n, G), twice)
    r.close()
    first.close()
    c.close()
