"""What a server of long contexts does with a cache beside plain decoding, one call at a time.

It drafts trees of tokens and verifies them in one pass (attention of a tree over the cache, then the accepted path
becomes the context), and it shrinks caches that grew too long (the attention weight that every position gets is added
up, and the lightest positions are evicted).  ``run`` makes those calls of the framework where ``own`` is set; otherwise
it computes the same with elementary tensor operations in 32 bits.

A case is a dict of plain values; ``kind`` says which call it times:
  tree    attention of drafted trees, one for each user: ``nodes`` tokens behind ``ctx`` positions (both comma-separated)
  accept  ``nodes`` drafted positions written behind ``n`` others, and ``path`` of them kept, in ``layers`` layers
  weigh   the attention weights of one query for each user (``window`` 0) or of a user's last ``window`` queries, added to
          what each cached position has so far
  evict   ``keep`` of ``n`` positions kept by their weight, in ``layers`` layers: the ``first`` and ``last`` ones and the
          heaviest of the others

A tree's tokens come parents first; ``parents`` holds each one's parent (-1: none, its parent is the last cached
position; -2: no token, a row that pads the batch).  A token attends to the cached positions, its ancestors and itself.
A 4-bit cache holds blocks of 32 values along a head as E2M1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign) times a
power of two: the exponent of the block's largest fp16 magnitude, rounded to one mantissa bit, less 2, in [-23, 13].
"""
import math
import random
import types

import torch

own = False

# hidden, query heads, kv heads, head dim
SHAPES = {
    "tiny": (512, 8, 2, 64),
    "8b": (4096, 32, 8, 128),
    "32b": (5120, 40, 8, 128),
    "70b": (8192, 64, 8, 128),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32
MAX_NODES = 256  # tokens of a tree
MAX_ROWS = 32  # queries of a weighing call


def _tree(name, shape, ctx, nodes, cache="f16", io="bf16", paged=False, pad=0):
    return {"name": name, "kind": "tree", "shape": shape, "ctx": ctx, "nodes": nodes, "cache": cache, "io": io,
            "paged": paged, "pad": pad}


def _accept(name, shape, n, nodes, path, layers, cache="f16", io="bf16", paged=False):
    return {"name": name, "kind": "accept", "shape": shape, "n": n, "nodes": nodes, "path": path, "layers": layers,
            "cache": cache, "io": io, "paged": paged}


def _weigh(name, shape, ctx, window=0, cache="f16", io="bf16", paged=False):
    return {"name": name, "kind": "weigh", "shape": shape, "ctx": ctx, "window": window, "cache": cache, "io": io,
            "paged": paged}


def _evict(name, shape, n, keep, first, last, layers, cache="f16", paged=False, inplace=False):
    return {"name": name, "kind": "evict", "shape": shape, "n": n, "keep": keep, "first": first, "last": last,
            "layers": layers, "cache": cache, "paged": paged, "inplace": inplace}


def listed():
    return [
        # a small model's single drafted token behind a short prompt: launches and little else
        _tree("tree_tiny_1", "tiny", "37", "1", io="f32"),
        # the usual draft of a chat turn: a small tree behind a few pages
        _tree("tree_8b_26_2k", "8b", "2000", "26"),
        # a full draft behind a long document
        _tree("tree_8b_64_32k", "8b", "32768", "64", paged=True),
        # four users of very different lengths, their trees padded to a batch, on a 4-bit cache
        _tree("tree_8b_b4_4bit", "8b", "16384,4096,1000,1", "48,7,64,17", cache="mxfp4", io="f16", paged=True, pad=3),
        # a wide draft of a large model, queries in 32 bits
        _tree("tree_70b_128_40k", "70b", "40001", "128", io="f32"),
        # the accepted tokens of a draft, in a slice of a model's layers
        _accept("accept_8b_60", "8b", 3001, 60, 5, 4),
        # the same of a wide draft in 4 bits, across pages
        _accept("accept_70b_200_4bit", "70b", 1999, 200, 70, 2, cache="mxfp4", io="f32", paged=True),
        # a decode step's weights of four users
        _weigh("weigh_8b_b4_32k", "8b", "32768,16384,8192,1024", cache="mxfp4", io="f32", paged=True),
        # the last queries of a long prompt, which say what of it will be needed
        _weigh("weigh_8b_16k_w32", "8b", "16384", window=32),
        # a small model's cache brought back to its budget
        _evict("evict_tiny_300", "tiny", 300, 200, 4, 64, 1),
        # a long prompt cut to a quarter, for a second user
        _evict("evict_8b_16k", "8b", 16384, 4096, 4, 512, 4),
        # the same in 4 bits and in place, from pages that another user shares
        _evict("evict_8b_32k_4bit_inplace", "8b", 32000, 8001, 4, 1000, 2, cache="mxfp4", paged=True, inplace=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _seconds(case):
    """A rough time of a case's work, to keep drawn cases below the largest listed one of their kind."""
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 0.8e15


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "accept", "weigh", "weigh", "evict", "evict"])
    most = max(_seconds(c) for c in listed() if c["kind"] == kind)
    while True:
        c = _draw(rng, kind)
        if _seconds(c) <= most:
            return c


def _draw(rng, kind):
    flag = lambda: rng.random() < 0.5  # noqa: E731
    shape = rng.choice(["tiny", "8b", "8b", "32b", "70b"])
    io = rng.choice(["f32", "bf16", "bf16", "f16"])
    cache = rng.choice(["f16", "f16", "mxfp4"])
    users = 1 if flag() else rng.randint(2, 4)
    if kind == "tree":
        ctx = [rng.choice([0, 1]) if rng.random() < 0.1 else _log_int(rng, 1, 65536) for _ in range(users)]
        nodes = [_log_int(rng, 1, MAX_NODES) for _ in range(users)]
        c = _tree("", shape, ",".join(map(str, ctx)), ",".join(map(str, nodes)), cache, io, flag(),
                  rng.randint(0, 3) if flag() else 0)
    elif kind == "accept":
        nodes = _log_int(rng, 1, MAX_NODES)
        c = _accept("", shape, _log_int(rng, 1, 5000) - 1, nodes, _log_int(rng, 1, nodes), rng.randint(1, 4), cache, io, flag())
    elif kind == "weigh":
        ctx = [_log_int(rng, 1, 65536) for _ in range(users)]
        c = _weigh("", shape, ",".join(map(str, ctx)), 0 if flag() else rng.randint(1, MAX_ROWS // users), cache, io, flag())
    else:
        n = _log_int(rng, 2, 32768)
        keep = _log_int(rng, 1, n)
        first = rng.randint(0, min(keep, 70))
        c = _evict("", shape, n, keep, first, rng.randint(0, keep - first), rng.randint(1, 4), cache, flag(), flag())
    c.pop("name", None)
    return c


# ---------------------------------------------------------------- inputs


def _ints(text):
    return [int(v) for v in text.split(",")]


def _spans(case):
    """A weighing call's queries: (user, positions that it attends to), a user's last queries in order."""
    w = max(case["window"], 1)
    return [(u, max(n - w + 1 + i, 0)) for u, n in enumerate(_ints(case["ctx"])) for i in range(w)]


def _parents(case, seed):
    """Each tree's parents: mostly a recent token, as drafts of a few continuations per step have them, some roots."""
    rng = random.Random(seed)
    trees = []
    for n in _ints(case["nodes"]):
        p = [-1 if rng.random() < 0.1 else max(i - 1 - int(rng.expovariate(0.2)), -1) for i in range(n)]
        for i in range(max(n - case["pad"], 1), n):
            p[i] = -2
        trees.append(p)
    return trees


def _path(case, seed):
    return sorted(random.Random(seed).sample(range(case["nodes"]), case["path"]))


def _inputs(case, seed):
    """Every input of a case, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    hidden, nq, nkv, hd = SHAPES[case["shape"]]

    def normal(shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)

    def saved(n, dtype=torch.bfloat16):  # keys and values at the scale that N(0, 0.02^2) projections of unit rows give
        return [normal((n, nkv, hd), 0.02 * math.sqrt(hidden), dtype) for _ in range(2)]

    kind = case["kind"]
    d = {}
    if kind == "tree":
        nodes = _ints(case["nodes"])
        d["kv"] = [saved(n + m) for n, m in zip(_ints(case["ctx"]), nodes)]
        d["q"] = normal((sum(nodes), nq, hd), 1.0, DTYPES[case["io"]])
        flat = [p for tree in _parents(case, seed) for p in tree]
        d["parents"] = torch.tensor(flat, dtype=torch.int32, device="cuda")
    elif kind == "accept":
        d["new"] = [saved(case["nodes"], DTYPES[case["io"]]) for _ in range(case["layers"])]
        d["path"] = _path(case, seed)
    elif kind == "weigh":
        lens = _ints(case["ctx"])
        d["kv"] = [saved(n) for n in lens]
        d["q"] = normal((len(_spans(case)), nq, hd), 1.0, DTYPES[case["io"]])
        d["prior"] = [torch.exp(normal((nkv, n), 1.5) - 8) for n in lens]
    else:
        n, layers = case["n"], case["layers"]
        d["kv"] = [saved(n) for _ in range(layers)]
        # weights over several orders of magnitude, some positions never looked at, and ties in every other layer
        w = torch.exp(normal((layers, nkv, n), 2.0))
        w = torch.where(torch.rand((layers, nkv, n), generator=g, device="cuda") < 0.1, 0.0, w)
        w[1::2] = w[1::2].bfloat16().float()
        d["weights"] = w
    return d


class _Held:
    """What a serving program holds: a stage whose layers' weights are not used here, and its cache."""

    def __init__(self, case, d):
        import numpy as np

        from paper_2609_34045_amd import stage as kf

        self.kv = None
        kind = case["kind"]
        _, nq, nkv, hd = SHAPES[case["shape"]]
        layers = case.get("layers", 1)
        shape = types.SimpleNamespace(n_layers=layers, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=hd, ffn=64,
                                      vocab=0, rms_eps=1e-5, rope_theta=1e4, qk_norm=False)
        sizes = {"attn_norm": 64, "mlp_norm": 64, "wq": nq * hd * 64, "wk": nkv * hd * 64, "wv": nkv * hd * 64,
                 "wo": 64 * nq * hd, "wg": 64 * 64, "wu": 64 * 64, "wd": 64 * 64}
        layer = {k: np.zeros(n, np.uint16) for k, n in sizes.items()}
        self.stage = kf.Stage(shape, 0, layers, lambda l: layer)
        if kind in ("tree", "weigh"):
            lens = [n + m for n, m in zip(_ints(case["ctx"]), _ints(case["nodes"]))] if kind == "tree" else _ints(case["ctx"])
        elif kind == "accept":
            lens = [case["n"] + case["nodes"]]
        else:
            lens = [case["n"], case["n"]]  # the second is the one that eviction makes
        pages = sum((n + 63) // 64 for n in lens)
        self.kv = self.stage.kv(len(lens), max(lens), pages if case["paged"] else None, dtype=case["cache"])
        if kind in ("weigh", "evict"):
            self.kv.track()
        if kind in ("tree", "weigh"):
            for u, (k, v) in enumerate(d["kv"]):
                self.kv.write(0, u, 0, k, v)
        elif kind == "accept":
            self.kv.set_len(0, case["n"])
        else:
            for l, (k, v) in enumerate(d["kv"]):
                self.kv.write(l, 0, 0, k, v)
                self.kv.set_weights(l, 0, 0, d["weights"][l])
            self.kv.set_len(0, case["n"])
        self.stage.sync()

    def __del__(self):
        if getattr(self, "kv", None) is not None:
            self.kv.close()
        if getattr(self, "stage", None) is not None:
            self.stage.close()


def prepare(case, seed):
    d = _inputs(case, seed)
    s = types.SimpleNamespace(case=case, d=d, held=None, rows=None)
    if own:
        s.held = _Held(case, d)
        for name in ("kv", "weights"):  # the cache holds them
            d.pop(name, None)
    elif "kv" in d:
        s.rows = [[_hold(t, case["cache"]) for t in kv] for kv in d.pop("kv")]
    return s


# ---------------------------------------------------------------- the framework's calls


def _run_own(s):
    case, d, kv = s.case, s.d, s.held.kv
    kind = case["kind"]
    if kind == "tree":
        lens = _ints(case["ctx"])
        return kv.attend_tree(0, list(range(len(lens))), lens, _ints(case["nodes"]), d["parents"], d["q"])
    if kind == "accept":
        n, layers = case["n"], range(case["layers"])
        for l in layers:
            kv.write(l, 0, n, *d["new"][l])
        kv.accept(0, n, d["path"])
        return [kv.read(l, 0, n, case["path"]) for l in layers]
    if kind == "weigh":
        lens = _ints(case["ctx"])
        for u, w in enumerate(d["prior"]):
            kv.set_weights(0, u, 0, w)
        spans = _spans(case)
        kv.weigh(0, [u for u, _ in spans], [n for _, n in spans], d["q"])
        return [kv.weights(0, u, 0, n) for u, n in enumerate(lens)]
    src = 0
    if case["inplace"]:
        kv.fork(0, 1)
        src = 1
    keep, layers = case["keep"], range(case["layers"])
    kept = kv.evict(src, 1, keep, case["first"], case["last"], kept=True)
    return {"kept": kept, "kv": [kv.read(l, 1, 0, keep) for l in layers],
            "weights": [kv.weights(l, 1, 0, keep) for l in layers]}


# ---------------------------------------------------------------- the same in plain tensor operations


def _hold(x, kind):
    """What a cache of this kind keeps of x [..., hd]: fp16, or packed 4-bit codes and their blocks' exponents."""
    x = x.half()
    if kind == "f16":
        return (x,)
    b = x.float().unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True).view(torch.int32)
    e = (((top + 0x200000) >> 23) - 129).clamp(-23, 13)
    y = torch.ldexp(b, -e)
    a = y.abs().clamp(max=6.0)
    code = torch.where(a < 2, (a * 2).round(), torch.where(a < 4, a.round() + 2, (a / 2).round() + 4)).to(torch.uint8)
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e.squeeze(-1) + 127).to(torch.uint8)


def _value(held):
    """The fp32 values that _hold's tensors stand for."""
    if len(held) == 1:
        return held[0].float()
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=held[0].device)
    table = torch.cat([table, -table])
    code = torch.stack([held[0] & 15, held[0] >> 4], -1).flatten(-2)
    v = table[code.int()].unflatten(-1, (-1, BLOCK))
    return torch.ldexp(v, held[1].int()[..., None] - 127).flatten(-2)


def _visible(parents):
    """[n, n] truth values: which tokens of its tree each one attends to."""
    n = parents.shape[0]
    real = parents > -2
    see = torch.diag(real)
    up = torch.where(parents >= 0, parents, n).long()  # n stands for no parent
    up = torch.cat([up, torch.full_like(up[:1], n)])
    see = torch.cat([see, torch.zeros_like(see[:1])])
    for _ in range(n.bit_length()):
        see = see | see[up]
        up = up[up]
    return see[:n]


def _scores(q, k):
    """[nkv, rows * group, L] fp32 scores of q [rows, nq, hd] over k [L, nkv, hd]."""
    rows, nq, hd = q.shape
    nkv = k.shape[1]
    group = nq // nkv
    qs = q.float().view(rows, nkv, group, hd).permute(1, 3, 0, 2).reshape(nkv, hd, rows * group)
    return torch.matmul(k.transpose(0, 1).contiguous(), qs).transpose(1, 2) / math.sqrt(hd)


def _probabilities(z, hidden):
    """Softmax over the last axis of z [nkv, rows, group, L] without the positions that hidden [rows, L] marks."""
    z = torch.where(hidden[:, None], -math.inf, z)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m > -math.inf, m, 0.0))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, 1.0)


def _tree_attention(q, k, v, ctx, parents):
    rows, nq, hd = q.shape
    nkv = k.shape[1]
    hidden = torch.cat([(parents < -1)[:, None].expand(rows, ctx), ~_visible(parents)], 1)
    p = _probabilities(_scores(q, k).unflatten(1, (rows, nq // nkv)), hidden)
    o = torch.matmul(p.flatten(1, 2), v.transpose(0, 1).contiguous())
    return o.unflatten(1, (rows, nq // nkv)).transpose(0, 1).reshape(rows, nq, hd).to(q.dtype)


def _heaviest(w, keep, first, last):
    """[..., keep] positions kept of w [..., n], in order; of equal weights the lower position is kept."""
    n = w.shape[-1]
    at = torch.arange(n, device=w.device)
    w = torch.where((at < first) | (at >= n - last), math.inf, w)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    return torch.sort(order, dim=-1).values


def _run_plain(s):
    case, d = s.case, s.d
    kind = case["kind"]
    if kind == "tree":
        out, at = [], 0
        for ctx, n, (k, v) in zip(_ints(case["ctx"]), _ints(case["nodes"]), s.rows):
            out.append(_tree_attention(d["q"][at:at + n], _value(k), _value(v), ctx, d["parents"][at:at + n]))
            at += n
        return torch.cat(out)
    if kind == "accept":
        path = torch.tensor(d["path"], device="cuda")
        return [tuple(_value([t[path] for t in _hold(x, case["cache"])]) for x in new) for new in d["new"]]
    if kind == "weigh":
        out, at, w = [], 0, max(case["window"], 1)
        spans = _spans(case)
        for (k, _), prior in zip(s.rows, d["prior"]):
            k, n = _value(k), prior.shape[1]
            seen = torch.tensor([m for _, m in spans[at:at + w]], device="cuda")
            z = _scores(d["q"][at:at + w], k)
            p = _probabilities(z.unflatten(1, (w, -1)), torch.arange(n, device="cuda") >= seen[:, None])
            out.append(prior + p.sum((1, 2)))
            at += w
        return out
    kept = _heaviest(d["weights"], case["keep"], case["first"], case["last"])
    nkv = kept.shape[1]
    head = torch.arange(nkv, device="cuda")
    kv = [tuple(_value([part[at.t(), head] for part in held]) for held in layer) for at, layer in zip(kept, s.rows)]
    weights = d["weights"].gather(2, kept)
    return {"kept": kept.to(torch.int32), "kv": kv, "weights": list(weights)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    """Inputs and cache read once, results written once; a multiply and an add per product."""
    kind = case["kind"]
    _, nq, nkv, hd = SHAPES[case["shape"]]
    row = 2 * nkv * hd * (2 if case["cache"] == "f16" else 17 / 32)  # a cached position's keys and values
    if kind == "tree":
        ctx, nodes = _ints(case["ctx"]), _ints(case["nodes"])
        return {"bytes": (sum(ctx) + sum(nodes)) * row + sum(nodes) * (2 * nq * hd * BYTES[case["io"]] + 4),
                "flops": 4.0 * nq * hd * sum(n * (c + 1) for c, n in zip(ctx, nodes))}
    if kind == "accept":  # written, the accepted ones moved and read
        values = 2 * nkv * hd
        return {"bytes": case["layers"] * (case["nodes"] * (values * BYTES[case["io"]] + row)
                                           + case["path"] * (3 * row + 4 * values)), "flops": 0}
    if kind == "weigh":  # keys alone; the weights given, and taken out again
        spans = _spans(case)
        return {"bytes": sum(_ints(case["ctx"])) * (row / 2 + 2 * nkv * 4) + len(spans) * nq * hd * BYTES[case["io"]],
                "flops": 2.0 * nq * hd * sum(n for _, n in spans)}
    n, keep = case["n"], case["keep"]
    return {"bytes": case["layers"] * (n * nkv * 4 + keep * (3 * row + 4 * 2 * nkv * hd + nkv * (4 + 3 * 4))), "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits


def _nearest(x, kind):
    """The value in 64 bits that a cache of this kind stands for: the nearest element, the even one of two as near."""
    x = x.to(torch.float16).to(torch.float64)
    if kind == "f16":
        return x
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    m, e = torch.frexp(b.abs().max(-1, keepdim=True).values)
    e = torch.where(m >= 0.875, e + 1, e) - 3
    e = torch.where(m == 0, -23, e).clamp(min=-23, max=13)
    scale = torch.exp2(e.to(torch.float64))
    size = (b / scale).abs()
    out = torch.zeros_like(size)
    magnitudes = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for i in range(1, 8):  # past the middle between two neighbours the upper one; on it, the one of even index
        middle = (magnitudes[i - 1] + magnitudes[i]) / 2
        out = torch.where((size > middle) if i % 2 else (size >= middle), magnitudes[i], out)
    return (torch.sign(b) * out * scale).reshape(x.shape)


def _softmax_of(q, k, see):
    """Probabilities [rows, L] of q [rows, hd] over k [L, hd] where see [rows, L] is set; a row of zeros where nothing is."""
    z = torch.where(see, (q.double() @ k.t().contiguous()) * k.shape[1] ** -0.5, -math.inf)
    return torch.nan_to_num(torch.softmax(z, -1), nan=0.0)


def exact(case, seed):
    d = _inputs(case, seed)
    kind = case["kind"]
    _, nq, nkv, hd = SHAPES[case["shape"]]
    if kind == "tree":
        out = []
        for tree, ctx, (k, v), at in zip(_parents(case, seed), _ints(case["ctx"]), d["kv"],
                                         torch.tensor([0] + _ints(case["nodes"])).cumsum(0).tolist()):
            n = len(tree)
            see = torch.zeros((n, ctx + n), dtype=torch.bool)
            for i, p in enumerate(tree):
                if p == -2:
                    continue
                see[i, :ctx] = True
                j = i
                while j >= 0:
                    see[i, ctx + j] = True
                    j = tree[j]
            see = see.cuda()
            k, v = (_nearest(t, case["cache"]) for t in (k, v))
            o = torch.empty((n, nq, hd), dtype=torch.float64, device="cuda")
            for h in range(nq):
                g = h // (nq // nkv)
                o[:, h] = _softmax_of(d["q"][at:at + n, h], k[:, g], see) @ v[:, g].contiguous()
            out.append(o)
        return torch.cat(out)
    if kind == "accept":
        return [tuple(_nearest(torch.stack([x[i] for i in d["path"]]), case["cache"]) for x in new) for new in d["new"]]
    if kind == "weigh":
        out = []
        for u, ((k, _), prior) in enumerate(zip(d["kv"], d["prior"])):
            k, w = _nearest(k, case["cache"]), prior.double()
            mine = [(i, n) for i, (user, n) in enumerate(_spans(case)) if user == u]
            see = torch.stack([torch.arange(k.shape[0], device="cuda") < n for _, n in mine])
            q = d["q"][[i for i, _ in mine]]
            for h in range(nq):
                w[h // (nq // nkv)] += _softmax_of(q[:, h], k[:, h // (nq // nkv)], see).sum(0)
            out.append(w)
        return out
    n, keep, first, last = case["n"], case["keep"], case["first"], case["last"]
    weights = d["weights"].cpu()
    kept = torch.empty((case["layers"], nkv, keep), dtype=torch.int64)
    for l in range(case["layers"]):
        for g in range(nkv):
            w = weights[l, g].tolist()
            others = sorted(range(first, n - last), key=lambda t: (-w[t], t))[:keep - first - last]
            kept[l, g] = torch.tensor(list(range(first)) + sorted(others) + list(range(n - last, n)))
    kept = kept.cuda()
    kv = [tuple(torch.stack([_nearest(x[:, g][at[g]], case["cache"]) for g in range(nkv)], 1) for x in layer)
          for at, layer in zip(kept, d["kv"])]
    taken = [torch.stack([d["weights"][l, g][kept[l, g]] for g in range(nkv)]).double() for l in range(case["layers"])]
    return {"kept": kept.to(torch.int32), "kv": kv, "weights": taken}
