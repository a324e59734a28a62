"""The work that is timed of a document's cache held in 8 bits.

Four operators: ``store`` (rows quantised as they are written into the cache, and the blocks they
fall into read back), ``attend`` (attention of query rows over such caches), ``weigh`` (the same
attention, which also leaves at every entry the weight that it got) and ``evict`` (the entries of
each layer and KV head with the largest weights chosen and kept, the others dropped).

The stored form: 64 consecutive entries of a layer and KV head are a block; its keys share one power
of two and its values another, the smallest with which the largest magnitude is at most 448; an
entry is a floating-point number of 4 exponent and 3 mantissa bits times that power.  While rows of a
block stay, its powers only rise: rows that stay are rounded again to the larger one.  Kept entries
form blocks of their own, with powers of their own.

Shapes are those of the presets of this repository (heads, KV heads, head size, layers), contexts
those of its workloads (512, 5000, 8192, 12345, 16384) and, for caches alone, longer ones.  A row
at position -1 sees no key.
"""
import math

import torch

own = False

# heads, KV heads, head size, layers of the presets
SHAPES = {
    "tiny": (4, 2, 64, 2),
    "llama8b": (32, 8, 128, 32),
    "qwen7b": (28, 4, 128, 28),
    "mistral7b": (32, 8, 128, 32),
}
BLOCK = 64
LARGEST = 448.0
LEAST = -100  # the smallest power of two of a block


# ------------------------------------------------------------------ cases

def listed():
    return [
        # One new position's rows, every layer: what a decoding step appends to its document.
        dict(name="store_token", op="store", preset="llama8b", dtype="bf16", layers=32, n=5000,
             rows=1, spread=False),
        # A whole document held after its prefill.
        dict(name="store_document_5000", op="store", preset="qwen7b", dtype="bf16", layers=28,
             n=5000, rows=5000, spread=False),
        # One query token over a long cache: a layer of a decoding step.
        dict(name="attend_token_131072", op="attend", preset="llama8b", dtype="bf16", docs=1,
             n=131072, rows=1, spread=False, empty=False),
        # A token for each of sixteen documents of an odd length, one of which sees no key yet.
        dict(name="attend_batch_16x8191", op="attend", preset="llama8b", dtype="bf16", docs=16,
             n=8191, rows=1, spread=True, empty=True),
        # The rows of a repair (span of 8 and a window of 32) against the document.
        dict(name="attend_repair_40", op="attend", preset="mistral7b", dtype="bf16", docs=1, n=5000,
             rows=40, spread=True, empty=False),
        # A chunk of a prefill at the end of a long document of odd length.
        dict(name="attend_chunk_4096", op="attend", preset="qwen7b", dtype="bf16", docs=1, n=12345,
             rows=4096, spread=False, empty=False),
        # The small fp32 model's rows, weighed; the smallest call.
        dict(name="weigh_tiny_fp32", op="weigh", preset="tiny", dtype="fp32", docs=1, n=500,
             rows=36, spread=True, empty=True),
        # One query token of a decoding step that gathers weights for a later eviction, 7 heads a
        # KV head.
        dict(name="weigh_token_5000", op="weigh", preset="qwen7b", dtype="bf16", docs=1, n=5000,
             rows=1, spread=False, empty=False),
        # The last rows of a document, by which its entries are judged before it is shortened.
        dict(name="weigh_window_64", op="weigh", preset="llama8b", dtype="bf16", docs=1, n=16384,
             rows=64, spread=False, empty=False),
        # A chunk of a prefill that gathers weights.
        dict(name="weigh_chunk_4096", op="weigh", preset="qwen7b", dtype="bf16", docs=1, n=12345,
             rows=4096, spread=False, empty=False),
        # The small fp32 model's document halved, its first four and last 32 entries protected.
        dict(name="evict_tiny_fp32", op="evict", preset="tiny", dtype="fp32", layers=2, n=512,
             keep=256, first=4, recent=32),
        # A long document of odd length cut to a third in every layer.
        dict(name="evict_document_12345", op="evict", preset="llama8b", dtype="bf16", layers=32,
             n=12345, keep=4096, first=4, recent=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    preset = rng.choice(["tiny", "llama8b", "qwen7b", "mistral7b"])
    dtype = "fp32" if rng.random() < (0.6 if preset == "tiny" else 0.15) else "bf16"
    op = rng.choice(["store", "attend", "attend", "weigh", "weigh", "evict"])
    if op in ("store", "evict"):
        layers = rng.randint(1, SHAPES[preset][3])
        if dtype == "fp32":
            layers = max(1, layers // 2)
        if op == "store":
            n = _log_int(rng, 1, 5000)
            rows = n if rng.random() < 0.4 else _log_int(rng, 1, n)
            return dict(op="store", preset=preset, dtype=dtype, layers=layers, n=n, rows=rows,
                        spread=rng.random() < 0.5)
        n = _log_int(rng, 2, 8192)
        keep = max(1, int(n * rng.uniform(0.05, 1.0)))
        first = min(keep, rng.choice([0, 1, 4, 16]))
        recent = int((keep - first) * rng.choice([0.0, 0.1, 0.5]))
        return dict(op="evict", preset=preset, dtype=dtype, layers=layers, n=n, keep=keep,
                    first=first, recent=recent)
    kind = rng.choice(["token", "token", "batch", "rows", "rows", "chunk"])
    case = dict(op=op, preset=preset, dtype=dtype, docs=1, n=_log_int(rng, 1, 131072), rows=1,
                spread=rng.random() < 0.5, empty=rng.random() < 0.3)
    if kind == "batch":
        case.update(docs=rng.randint(2, 16), n=_log_int(rng, 16, 8191), rows=rng.choice([1, 1, 2, 3]))
    elif kind == "rows" or (kind == "chunk" and dtype == "fp32"):
        n = _log_int(rng, 64, 16384)
        case.update(n=n, rows=min(n, _log_int(rng, 2, 64)))
    elif kind == "chunk":
        n = _log_int(rng, 512, 12345)
        case.update(n=n, rows=min(n, _log_int(rng, 65, 4096)))
    if case["docs"] * case["rows"] == 1:
        case["empty"] = False
    return case


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _positions(g, case):
    """Positions [docs, rows] of a case's rows, ascending, the last of the document among them."""
    n, rows, docs = case["n"], case["rows"], case.get("docs", 1)
    if not case["spread"]:
        return torch.arange(n - rows, n, dtype=torch.int32, device="cuda").expand(docs, rows)
    at = torch.rand(docs, n, generator=g, device="cuda")
    at[:, n - 1] = 2.0
    return at.topk(rows, dim=1).indices.sort(dim=1).values.to(torch.int32)


def _key_value_rows(g, shape, dtype):
    """K and V rows [..., heads, head size] as a trained model has them: some key entries
    (channels) are much larger than the rest, and rows differ in size from position to position."""
    out = []
    for which in range(2):
        x = torch.randn(shape, generator=g, device="cuda")
        channel = torch.exp(0.7 * torch.randn(shape[-2:], generator=g, device="cuda"))
        size = torch.exp(0.3 * torch.randn((shape[0],) + (1,) * (len(shape) - 1), generator=g,
                                           device="cuda"))
        x *= size
        if which == 0:
            x *= channel
        out.append(x.to(dtype))
    return out


def _inputs(case, seed):
    """Device tensors, from the seed alone."""
    H, G, dh, _ = SHAPES[case["preset"]]
    g = _generator(seed)
    dt = _torch_dtype(case)
    n = case["n"]
    if case["op"] in ("store", "evict"):
        L = case["layers"]
        doc = _key_value_rows(g, (n, L, G, dh), dt)  # the document as it stands before the call
        if case["op"] == "store":
            pos = _positions(g, case)[0]
            k, v = _key_value_rows(g, (case["rows"], L, G, dh), dt)
            return dict(doc=doc, pos=pos, k=k, v=v)
        # a few entries carry most of the weight, and some none at all
        w = torch.exp(1.5 * torch.randn((L, G, n), generator=g, device="cuda"))
        w *= torch.rand((L, G, n), generator=g, device="cuda") > 0.1
        return dict(doc=doc, weight=w)
    D, R = case["docs"], case["rows"]
    pos = _positions(g, case).clone()
    if case["empty"]:
        pos[0, 0] = -1
    k, v = _key_value_rows(g, (D * n, G, dh), dt)
    q = (torch.randn((D, R, H, dh), generator=g, device="cuda") * 1.5).to(dt)
    return dict(pos=pos, k=k.view(D, n, G, dh), v=v.view(D, n, G, dh), q=q)


class _Kept:
    """What the process keeps between calls: its models."""
    models = {}


def _model(case):
    """The handle whose shape, stream and workspaces the caches use; its weights take no part."""
    from paper_2609_17983_gb300 import kvrepair as kv
    from paper_2609_17983_gb300 import synth
    layers = case.get("layers", 1)
    key = (case["preset"], layers, case["dtype"])
    if key not in _Kept.models:
        if not _Kept.models:
            kv.use_torch_allocator()
        cfg = synth.preset(case["preset"], n_layers=layers, dtype=case["dtype"], vocab=1024, ffn=688)
        m = kv.Model(cfg, None, seed=0, max_context=1024, max_rows=64)
        m.set_stream(torch.cuda.current_stream().cuda_stream)
        _Kept.models[key] = m
    return _Kept.models[key]


def _touched(pos, n):
    """The entries of the blocks that these positions fall into."""
    hit = torch.zeros(-(-n // BLOCK), dtype=torch.bool, device=pos.device)
    hit[torch.div(pos.long(), BLOCK, rounding_mode="floor")] = True
    return hit.repeat_interleave(BLOCK)[:n].nonzero().squeeze(1)


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    H, G, dh, _ = SHAPES[case["preset"]]
    n, dt = case["n"], _torch_dtype(case)
    every = torch.arange(n).numpy()
    if case["op"] in ("store", "evict"):
        L = case["layers"]
        k, v = st.pop("doc")
        if case["op"] == "store":
            st["back"] = _touched(st["pos"], n)
            rows = len(st["back"])
        else:
            rows = case["keep"]
        if not own:
            st["held"] = [_quantise(x) for x in (k, v)]
            return st
        m = _model(case)
        st["cache"] = m.cache8(n)
        st["cache"].write(every, k, v)
        st["out"] = [torch.empty((rows, L, G, dh), dtype=dt, device="cuda") for _ in range(2)]
        if case["op"] == "store":
            st["at"] = st["pos"].cpu().numpy()
            st["back"] = st["back"].cpu().numpy()
        else:
            st["cache"].set_weights(st["weight"])
            st["into"] = m.cache8(rows)
            st["at"] = torch.arange(rows).numpy()
            st["kept"] = torch.empty((L, G, rows), dtype=torch.int32, device="cuda")
            st["number"] = torch.empty((L, G, rows), dtype=torch.int32, device="cuda")
            st["left"] = torch.empty((L, G, rows), dtype=torch.float32, device="cuda")
        return st
    k, v = st.pop("k"), st.pop("v")
    if not own:
        st["held"] = [_quantise(x.transpose(0, 1)) for x in (k, v)]
        return st
    D = case["docs"]
    m = _model(case)
    st["docs"] = [m.cache8(n) for _ in range(D)]
    for d, doc in enumerate(st["docs"]):
        doc.write(every, k[d].unsqueeze(1), v[d].unsqueeze(1))
    st["rows"] = m.rows8(list(zip(st["docs"], st["pos"].cpu().numpy())))
    st["out"] = torch.empty_like(st["q"])
    if case["op"] == "weigh":
        st["weight"] = torch.empty((D, 1, G, n), dtype=torch.float32, device="cuda")
        st["number"] = torch.empty((D, 1, G, n), dtype=torch.int32, device="cuda")
    return st


# ------------------------------------------------------------------ the plain form

def _blocks(x):
    """[n, ...] as [blocks, 64, ...], zeros behind the last."""
    pad = -x.shape[0] % BLOCK
    if pad:
        x = torch.cat((x, torch.zeros((pad,) + x.shape[1:], dtype=x.dtype, device=x.device)))
    return x.view((-1, BLOCK) + x.shape[1:])


def _power(a):
    """Exponent of the smallest power of two t with a <= 448 t."""
    m, e = torch.frexp(a)
    return torch.where(a > 0, e - 9 + (m > 0.875).int(), LEAST).clamp(min=LEAST)


def _code(x, e):
    """Codes of values [blocks, 64, ..., head size] under the exponents e [blocks, ...]."""
    t = torch.exp2(-e.float()).unsqueeze(1).unsqueeze(-1)
    return (x * t).to(torch.float8_e4m3fn)


def _quantise(x):
    """Rows [n, ..., head size] as codes [blocks, 64, ..., head size] and exponents [blocks, ...]."""
    x = _blocks(x).float()
    e = _power(x.abs().amax(-1).amax(1))
    return [_code(x, e), e]


def _values(held):
    """fp32 values [n, ..., head size] of codes and exponents."""
    code, e = held
    return (code.float() * torch.exp2(e.float()).unsqueeze(1).unsqueeze(-1)).flatten(0, 1)


def _write(held, at, x, n):
    """Rows x into the positions at of a document of n."""
    blocks, slot = torch.unique(torch.div(at, BLOCK, rounding_mode="floor"), return_inverse=True)
    code, e = held[0][blocks], held[1][blocks]
    new = torch.zeros(code.shape[:2], dtype=torch.bool, device=at.device)
    new[slot, at % BLOCK] = True
    there = blocks.unsqueeze(1) * BLOCK + torch.arange(BLOCK, device=at.device) < n
    others = (there & ~new).any(1).view((-1,) + (1,) * (e.dim() - 1))
    value = _values((code, e)).view(code.shape)
    value[slot, at % BLOCK] = x.float()
    top = (value * new.view(new.shape + (1,) * (value.dim() - 2))).abs().amax(-1).amax(1)
    e = torch.maximum(_power(top), torch.where(others, e, LEAST))
    held[0][blocks], held[1][blocks] = _code(value, e), e


def _attend(q, pos, k, v):
    """softmax(q k / sqrt(head size)) v over the keys up to a row's position, and the weights of
    each key, summed over rows and the heads of its KV head: [docs, 1, KV heads, n]."""
    D, R, H, dh = q.shape
    n, G = k.shape[1:3]
    x = q.float().unflatten(2, (G, -1)).permute(0, 2, 3, 1, 4)  # [D, G, heads, R, dh]
    score = torch.matmul(x, k.permute(0, 2, 3, 1).unsqueeze(2)) * (1.0 / math.sqrt(dh))
    mask = (torch.arange(n, device=q.device) <= pos.unsqueeze(-1)).view(D, 1, 1, R, n)
    score.masked_fill_(~mask, -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = weight.sum(-1, keepdim=True)
    total = torch.where(total > 0, total, torch.ones_like(total))
    out = torch.matmul(weight, v.permute(0, 2, 1, 3).unsqueeze(2)) / total
    weight /= total
    return (out.permute(0, 3, 1, 2, 4).reshape(D, R, H, dh).to(q.dtype),
            weight.sum(3).sum(2).unsqueeze(1))


def _choose(weight, keep, first, recent):
    """Entries [..., keep] to keep of [..., n]: the first, the recent and those of most weight."""
    n = weight.shape[-1]
    at = torch.arange(n, device=weight.device)
    rank = torch.where((at < first) | (at >= n - recent), torch.full_like(weight, math.inf), weight)
    order = torch.argsort(rank, dim=-1, descending=True, stable=True)[..., :keep]
    return order.sort(-1).values.to(torch.int32)


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        if op == "store":
            st["cache"].write(st["at"], st["k"], st["v"])
            st["cache"].read(st["back"], *st["out"])
            return {"k": st["out"][0], "v": st["out"][1]}
        if op == "evict":
            st["cache"].choose(st["kept"], first=case["first"], recent=case["recent"])
            st["cache"].keep(st["kept"], into=st["into"])
            st["into"].read(st["at"], *st["out"])
            st["into"].entries(st["number"], st["left"])
            return {"kept": st["kept"], "k": st["out"][0], "v": st["out"][1],
                    "number": st["number"], "weight": st["left"]}
        if op == "attend":
            st["rows"].attention(0, st["q"], st["out"])
            return {"out": st["out"]}
        st["rows"].attention(0, st["q"], st["out"], weigh=0.0)
        for doc, number, weight in zip(st["docs"], st["number"], st["weight"]):
            doc.entries(number, weight)
        return {"out": st["out"], "weight": st["weight"]}
    dt = _torch_dtype(case)
    if op == "store":
        out = []
        for held, x in zip(st["held"], (st["k"], st["v"])):
            _write(held, st["pos"].long(), x, case["n"])
            out.append(_values(held)[st["back"]].to(dt))
        return {"k": out[0], "v": out[1]}
    if op == "evict":
        kept = _choose(st["weight"], case["keep"], case["first"], case["recent"])
        at = kept.long().permute(2, 0, 1)  # [keep, layers, KV heads]
        out = []
        for held in st["held"]:
            x = _values(held)
            x = torch.gather(x, 0, at.unsqueeze(-1).expand(at.shape + x.shape[-1:]))
            out.append(_values(_quantise(x))[:case["keep"]].to(dt))
        return {"kept": kept, "k": out[0], "v": out[1], "number": kept.clone(),
                "weight": torch.gather(st["weight"], 2, kept.long())}
    k, v = (_values(x)[:case["n"]].transpose(0, 1) for x in st["held"])
    out, weight = _attend(st["q"], st["pos"], k, v)
    return {"out": out} if op == "attend" else {"out": out, "weight": weight}


# ------------------------------------------------------------------ the same in 64 bits

def _exact_powers(x):
    """Per block of rows [n, ..., head size]: the smallest 2^e (e >= -100) with every magnitude at
    most 448 2^e, by doubling and halving from an estimate."""
    top = torch.stack([b.abs().amax(0).amax(-1) for b in x.split(BLOCK)])
    t = torch.exp2(torch.floor(torch.log2(top.clamp(min=1e-300) / LARGEST)))
    t = torch.where(top > LARGEST * t, 2 * t, t)
    t = torch.where(top <= LARGEST * t / 2, t / 2, t)
    return t.clamp(min=2.0 ** LEAST)


def _exact_codes(x, t):
    """Values nearest to rows x of blocks with powers t among +-(8 + m) 2^(p - 3) t, ties to even m;
    below the normal numbers whole steps of 2^-9 t."""
    t = t.repeat_interleave(BLOCK, 0)[:len(x)].unsqueeze(-1)
    y = x / t
    step = torch.full_like(y, 2.0 ** -9)
    for p in range(-5, 9):
        step = torch.where(y.abs() >= 2.0 ** p, torch.full_like(y, 2.0 ** (p - 3)), step)
    low = torch.floor(y / step)
    part = y / step - low
    up = (part > 0.5) | ((part == 0.5) & (torch.remainder(low, 2) == 1))
    return (low + up.double()) * step * t


def exact(case, seed):
    st = _inputs(case, seed)
    n = case["n"]
    if case["op"] == "store":
        out = []
        pos = st["pos"].long()
        for doc, x in zip(st["doc"], (st["k"], st["v"])):
            doc, x = doc.double(), x.double()
            was = _exact_powers(doc)
            held = _exact_codes(doc, was)
            fresh = torch.zeros_like(held)
            fresh[pos] = x
            new = torch.zeros(n, dtype=torch.bool, device="cuda")
            new[pos] = True
            gone = torch.stack([b.all() for b in new.split(BLOCK)])  # no row of the block stays
            was[gone] = 2.0 ** LEAST
            held[pos] = x
            held = _exact_codes(held, torch.maximum(was, _exact_powers(fresh)))
            out.append(held[_touched(pos, n)])
        return {"k": out[0], "v": out[1]}
    if case["op"] == "evict":
        L, G, _ = st["weight"].shape
        mid = st["weight"].double().clone()
        mid[..., :case["first"]] = math.inf
        mid[..., n - case["recent"]:] = math.inf
        # the keep-th largest, and of those equal to it the lowest ones
        edge = mid.sort(-1, descending=True).values[..., case["keep"] - 1:case["keep"]]
        above, same = mid > edge, mid == edge
        some = case["keep"] - above.sum(-1, keepdim=True)
        took = above | (same & (same.long().cumsum(-1) <= some))
        kept = took.nonzero()[:, 2].view(L, G, case["keep"])
        out = []
        for doc in st["doc"]:
            held = []
            for l in range(L):  # layer by layer: 64 bits of a whole document are many
                x = doc[:, l].double()
                x = _exact_codes(x, _exact_powers(x))
                x = torch.stack([x[kept[l, g], g] for g in range(G)], 1)
                held.append(_exact_codes(x, _exact_powers(x)))
            out.append(torch.stack(held, 1))
        kept32 = kept.to(torch.int32)
        return {"kept": kept32, "k": out[0], "v": out[1], "number": kept32,
                "weight": torch.gather(st["weight"], 2, kept).double()}
    H, G, dh, _ = SHAPES[case["preset"]]
    D, R, grp = case["docs"], case["rows"], H // G
    out = torch.zeros((D, R, H, dh), dtype=torch.float64, device="cuda")
    weight = torch.zeros((D, 1, G, n), dtype=torch.float64, device="cuda")
    for d in range(D):
        k, v = (_exact_codes(x, _exact_powers(x)) for x in (st["k"][d].double(), st["v"][d].double()))
        for g in range(G):
            for r0 in range(0, R, 512):
                q = st["q"][d, r0:r0 + 512, g * grp:(g + 1) * grp].double()
                x = torch.einsum("rhc,nc->rhn", q, k[:, g]) / math.sqrt(dh)
                hide = torch.arange(n, device="cuda")[None] > st["pos"][d, r0:r0 + 512, None]
                w = torch.softmax(x.masked_fill(hide[:, None], -math.inf), -1).nan_to_num(0.0)
                out[d, r0:r0 + 512, g * grp:(g + 1) * grp] = torch.einsum("rhn,nc->rhc", w, v[:, g])
                weight[d, 0, g] += w.sum((0, 1))
    return {"out": out} if case["op"] == "attend" else {"out": out, "weight": weight}


# ------------------------------------------------------------------ floors

def work(case):
    H, G, dh, _ = SHAPES[case["preset"]]
    es = 2 if case["dtype"] == "bf16" else 4
    n = case["n"]
    if case["op"] == "store":
        rows = case["rows"]
        blocks = -(-rows // BLOCK)  # at least; scattered rows read more of them back
        entries = 2 * case["layers"] * G * dh
        back = min(n, blocks * BLOCK)
        # rows in, codes written, the blocks' codes read, values out
        return {"bytes": entries * (rows * (es + 1) + back * (1 + es)),
                "flops": entries * (rows + back)}
    if case["op"] == "evict":
        keep, heads = case["keep"], case["layers"] * G
        # weights read; the list, codes, numbers and weights of what is kept written; kept codes
        # read, and again to give the values out; numbers and weights out
        return {"bytes": heads * (n * 4 + keep * (4 + 8 * 2 + 2 * dh * (3 + es))),
                "flops": heads * (n + keep * 4 * dh)}
    D, R = case["docs"], case["rows"]
    keys = n if R == 1 else n - (R - 1) / 2 if not case["spread"] else n * (R + 1) / (2 * R)
    io = 2 * D * R * H * dh * es
    flops = D * R * keys * H * dh * 4
    bytes_ = D * n * 2 * G * dh + io
    if case["op"] == "weigh":
        bytes_ += D * n * G * 4
        flops += D * R * keys * H * 2
    return {"bytes": bytes_, "flops": flops}
