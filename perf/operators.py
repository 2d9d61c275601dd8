"""What serving several continuations of long prompts needs beside a decode step, one call at a time.

A server that keeps beams, samples or users of long contexts scores tokens (log probabilities, their entropy and the
top alternatives), holds the cache in 4 bits, attends to it, moves users between caches and lets several users share
one prompt.  ``run`` makes those calls of the framework where ``own`` is set; otherwise it computes the same with
elementary tensor operations in 32 bits.

A case is a dict of plain values; ``kind`` says which call it times:
  head    log probabilities of ``rows`` hidden rows through the unembedding, with ``top`` alternatives
  logits  log probabilities of ``rows`` rows of logits that the program holds (some of them masked)
  attend  attention of one query row for each user over its cached positions, ``ctx`` (comma-separated)
  cache   ``n`` positions written into a 4-bit cache and read back
  copy    ``n`` positions of a user copied from a cache of one type into a cache of another, and read there
  fork    a prompt of ``n`` positions shared by ``users`` users, one new position for each, and attention of all

The 4-bit cache holds blocks of 32 values along a head as E2M1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign) times
a power of two: the exponent of the block's largest fp16 magnitude, rounded to one mantissa bit, less 2, in [-23, 13].
"""
import math
import types

import torch

own = False

# hidden, query heads, kv heads, head dim, vocab
SHAPES = {
    "tiny": (512, 8, 2, 64, 1000),
    "qwen3_tiny": (384, 8, 2, 64, 1000),
    "8b": (4096, 32, 8, 128, 128256),
    "32b": (5120, 40, 8, 128, 152064),
    "70b": (8192, 64, 8, 128, 128256),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BLOCK = 32
LAYERS = 2  # layers that a copy moves


def _head(name, shape, rows, top, io):
    return {"name": name, "kind": "head", "shape": shape, "rows": rows, "top": top, "io": io}


def _logits(name, vocab, rows, top, pad):
    return {"name": name, "kind": "logits", "vocab": vocab, "rows": rows, "top": top, "pad": pad}


def _attend(name, shape, ctx, cache="mxfp4", io="bf16", paged=False):
    return {"name": name, "kind": "attend", "shape": shape, "ctx": ctx, "cache": cache, "io": io, "paged": paged}


def _cache(name, shape, n, pos0=0, io="bf16", paged=False):
    return {"name": name, "kind": "cache", "shape": shape, "n": n, "pos0": pos0, "io": io, "paged": paged}


def _copy(name, shape, n, pos0=0, src="f16", dst="mxfp4"):
    return {"name": name, "kind": "copy", "shape": shape, "n": n, "pos0": pos0, "src": src, "dst": dst}


def _fork(name, shape, n, users=4, cache="mxfp4", io="bf16", paged=True):
    return {"name": name, "kind": "fork", "shape": shape, "n": n, "users": users, "cache": cache, "io": io,
            "paged": paged}


def listed():
    return [
        # a small model's token for one user, with the alternatives a beam needs: launches and little else
        _head("head_tiny_b1_top5", "tiny", 1, 5, "f32"),
        # one step of four beams of an 8B model: the head's weights are read once, five alternatives each
        _head("head_8b_b4_top5", "8b", 4, 5, "bf16"),
        # scoring a ragged chunk of a prompt (log likelihood and entropy of every given token)
        _head("head_8b_200", "8b", 200, 0, "bf16"),
        # a batch of logits that a sampler has masked (banned tokens, one row with nothing left), twenty alternatives a row
        _logits("logits_256_top20", 151936, 256, 20, 0),
        # an ordinary chat turn of one user: a few pages of cache, latency counts
        _attend("attend_8b_b1_200", "8b", "200"),
        # four users of very different lengths on one card
        _attend("attend_8b_b4_32k", "8b", "32768,16384,8192,1024", io="f32", paged=True),
        # two long documents under a large model's heads
        _attend("attend_70b_b2_128k", "70b", "131072,100001"),
        # a short remembered prefix put into a 4-bit cache, at an odd position
        _cache("cache_tiny_37", "tiny", 37, pos0=5, io="f32"),
        # restoring a saved prefix of 16384 positions into a 4-bit cache, and saving it back
        _cache("cache_8b_16k", "8b", 16384, io="bf16", paged=True),
        # a user that went idle: its fp16 cache moved into 4 bits
        _copy("copy_8b_8k_to_4bit", "8b", 8192),
        # four beams of one long prompt: shared pages, a position of its own for each, and their attention
        _fork("fork_8b_16k", "8b", 16001),
        # two samples of a short prompt in reserved fp16 caches
        _fork("fork_8b_300_f16", "8b", 300, users=2, cache="f16", paged=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _seconds(case):
    """A rough time of a case's work, to keep drawn cases below the largest listed one of their kind."""
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 0.8e15


def draw(rng):
    kind = rng.choice(["head", "logits", "attend", "attend", "cache", "copy", "fork"])
    most = max(_seconds(c) for c in listed() if c["kind"] == kind)
    while True:
        c = _draw(rng, kind)
        if _seconds(c) <= most:
            return c


def _draw(rng, kind):
    flag = lambda: rng.random() < 0.5  # noqa: E731
    shape = rng.choice(["tiny", "8b", "8b", "32b", "70b"])
    io = rng.choice(["f32", "bf16", "f16"])
    if kind == "head":
        rows = rng.randint(1, 4) if flag() else _log_int(rng, 5, 200)
        # alternatives of many rows of random logits have near ties, which any order of summation breaks its own way
        c = _head("", rng.choice(["tiny", "qwen3_tiny", "8b"]), rows, rng.randint(0, 6) if rows <= 4 else 0,
                  rng.choice(["f32", "bf16"]))
    elif kind == "logits":
        c = _logits("", _log_int(rng, 100, 262144), _log_int(rng, 1, 300), rng.randint(0, 32), rng.randint(0, 9))
    elif kind == "attend":
        ctx = ",".join(str(rng.choice([0, 1]) if rng.random() < 0.1 else _log_int(rng, 1, 131072))
                       for _ in range(rng.randint(1, 4)))
        cache = rng.choice(["mxfp4", "mxfp4", "f16"])
        c = _attend("", shape, ctx, cache, "bf16" if cache == "f16" else io, flag())
    elif kind == "cache":
        c = _cache("", shape, _log_int(rng, 1, 16384), rng.randint(0, 200), io, flag())
    elif kind == "copy":
        src, dst = rng.choice([("f16", "mxfp4"), ("mxfp4", "f16"), ("mxfp4", "mxfp4"), ("f16", "f16")])
        c = _copy("", shape, _log_int(rng, 1, 8192), rng.randint(0, 200), src, dst)
    else:
        cache = rng.choice(["mxfp4", "mxfp4", "f16"])
        c = _fork("", shape, _log_int(rng, 1, 16384), rng.randint(2, 4), cache, "bf16" if cache == "f16" else io,
                  flag())
    c.pop("name", None)
    return c


# ---------------------------------------------------------------- inputs


def _contexts(case):
    return [int(v) for v in case["ctx"].split(",")]


def _generator(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)

    return g, normal


def _saved(case, normal, n):
    """Keys and values of n positions at the scale that N(0, 0.02^2) projections of unit rows give them."""
    hidden, _, nkv, hd, _ = SHAPES[case["shape"]]
    std = 0.02 * math.sqrt(hidden)
    return [normal((n, nkv, hd), std, DTYPES[case.get("io", "bf16")]) for _ in range(2)]


def _inputs(case, seed):
    """Every input of a case, on the GPU, from the seed alone."""
    g, normal = _generator(case, seed)
    kind = case["kind"]
    d = {}
    if kind == "head":
        hidden, _, _, _, vocab = SHAPES[case["shape"]]
        rows = case["rows"]
        d["lm_head"] = normal((vocab, hidden), 0.02, torch.bfloat16)
        # gains of three significant bits: their products with the bf16 weights fit the 11 bits of the fp16 matrix a
        # stage folds them into, so that the errors measured are the call's own and not that rounding's
        steps = torch.tensor([0.75, 0.875, 1.0, 1.25, 1.5], device="cuda")
        d["gain"] = steps[torch.randint(0, 5, (hidden,), generator=g, device="cuda")].to(torch.bfloat16)
        d["targets"] = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
        # rows lean towards their token by anything between not at all and near certainty, as a model's do
        w = d["lm_head"][d["targets"].long()].float()
        lean = torch.rand((rows, 1), generator=g, device="cuda") * 16 / (0.02 * math.sqrt(hidden))
        d["hidden"] = (normal((rows, hidden)) + lean * w / w.norm(dim=-1, keepdim=True)).to(DTYPES[case["io"]])
    elif kind == "logits":
        rows, vocab = case["rows"], case["vocab"]
        z = torch.zeros((rows, vocab + case["pad"]), device="cuda")
        z[:, :vocab] = normal((rows, vocab), 3.0)
        banned = torch.rand((rows, vocab), generator=g, device="cuda") < 0.1
        if rows > 2:
            banned[rows // 2] = True  # a row that its masks leave empty
            z[rows - 1, :vocab] = z[rows - 1, :vocab].round()  # and one full of ties
        z[:, :vocab].masked_fill_(banned, -math.inf)
        d["logits"] = z[:, :vocab]  # the row stride is longer than a row where there is padding
        d["targets"] = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    elif kind in ("attend", "fork"):
        _, nq, _, hd, _ = SHAPES[case["shape"]]
        lens = _contexts(case) if kind == "attend" else [case["n"]]
        users = len(lens) if kind == "attend" else case["users"]
        d["kv"] = [[t.to(torch.bfloat16) for t in _saved(case, normal, n)] for n in lens]
        d["q"] = normal((users, nq, hd), 1.0, DTYPES[case["io"]])
        if kind == "fork":
            d["new"] = [_saved(case, normal, 1) for _ in range(users)]
    elif kind == "cache":
        d["kv"] = [_saved(case, normal, case["n"])]
    else:
        d["kv"] = [_saved(case, normal, case["n"]) for _ in range(LAYERS)]
    return d


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view("uint16")


class _Held:
    """What a serving program holds: a stage whose layers' weights are not used here, and its caches."""

    def __init__(self, case, d):
        import numpy as np

        from paper_2609_34045_amd import stage as kf

        self.caches = []
        kind = case["kind"]
        hidden, nq, nkv, hd, vocab = SHAPES.get(case.get("shape"), (64, 1, 1, 64, case.get("vocab")))
        layers = LAYERS if kind == "copy" else 1
        if kind not in ("head", "logits"):
            hidden, vocab = 64, 0
        elif kind == "logits":
            hidden = 64
        else:
            nq = nkv
        shape = types.SimpleNamespace(n_layers=layers, hidden=hidden, n_q_heads=nq, n_kv_heads=nkv, head_dim=hd, ffn=64,
                                      vocab=vocab, rms_eps=EPS, rope_theta=1e4, qk_norm=False)
        sizes = {"attn_norm": hidden, "mlp_norm": hidden, "wq": nq * hd * hidden, "wk": nkv * hd * hidden,
                 "wv": nkv * hd * hidden, "wo": hidden * nq * hd, "wg": 64 * hidden, "wu": 64 * hidden, "wd": hidden * 64}
        layer = {k: np.zeros(n, np.uint16) for k, n in sizes.items()}
        head = None
        if kind == "head":
            head = {"embed": np.zeros(vocab * hidden, np.uint16), "final_norm": _bits(d["gain"]),
                    "lm_head": _bits(d["lm_head"])}
        self.stage = kf.Stage(shape, 0, layers, lambda l: layer, head)
        if kind in ("head", "logits"):
            return
        pages = lambda n: (n + 63) // 64  # noqa: E731
        if kind == "attend":
            lens = _contexts(case)
            longest = max(max(lens), 1)
            self._cache(len(lens), longest, sum(max(1, pages(n)) for n in lens) if case["paged"] else None, case["cache"])
        elif kind == "fork":
            n = case["n"]
            self._cache(case["users"], n + 1, pages(n + 1) + 2 * case["users"] if case["paged"] else None, case["cache"])
        elif kind == "cache":
            n = case["pos0"] + case["n"]
            self._cache(1, n, pages(n) if case["paged"] else None, "mxfp4")
        else:
            for t in (case["src"], case["dst"]):
                self._cache(1, case["pos0"] + case["n"], None, t)
        if kind in ("attend", "fork"):
            for u, (k, v) in enumerate(d["kv"]):
                self.caches[0].write(0, u, 0, k, v)
                self.caches[0].set_len(u, k.shape[0])
        elif kind == "copy":
            for l, (k, v) in enumerate(d["kv"]):
                self.caches[0].write(l, 0, case["pos0"], k, v)
        self.stage.sync()

    def _cache(self, users, longest, pages, dtype):
        self.caches.append(self.stage.kv(users, longest, pages, dtype=dtype))

    def __del__(self):
        for kv in getattr(self, "caches", ()):
            kv.close()
        if getattr(self, "stage", None) is not None:
            self.stage.close()


def prepare(case, seed):
    d = _inputs(case, seed)
    s = types.SimpleNamespace(case=case, d=d, held=None, rows=None)
    if own:
        s.held = _Held(case, d)
        if case["kind"] == "head":
            d["lm_head"] = None  # the stage holds it
        if case["kind"] in ("attend", "fork", "copy"):
            d["kv"] = None  # the cache holds them
    elif case["kind"] in ("attend", "fork", "copy"):
        held = case["src"] if case["kind"] == "copy" else case["cache"]
        s.rows = [[_hold(t, held) for t in kv] for kv in d["kv"]]
        d["kv"] = None
    return s


# ---------------------------------------------------------------- the framework's calls


def _run_own(s):
    case, d, stage = s.case, s.d, s.held.stage
    kind = case["kind"]
    if kind == "head":
        return _scores(stage.head_logprobs(d["hidden"], d["targets"], top=case["top"]))
    if kind == "logits":
        return _scores(stage.logits_logprobs(d["logits"], d["targets"], top=case["top"]))
    kv = s.held.caches[0]
    if kind == "attend":
        lens = _contexts(case)
        return kv.attend(0, list(range(len(lens))), lens, d["q"])
    if kind == "cache":
        kv.write(0, 0, case["pos0"], *d["kv"][0])
        return kv.read(0, 0, case["pos0"], case["n"])
    if kind == "copy":
        to = s.held.caches[1]
        to.copy(kv, 0, 0, case["pos0"], case["n"])
        return [to.read(l, 0, case["pos0"], case["n"]) for l in range(LAYERS)]
    n, users = case["n"], list(range(case["users"]))
    for u in users[1:]:
        kv.fork(0, u, n)
    for u in users:
        kv.write(0, u, n, *d["new"][u])
    return kv.attend(0, users, [n + 1] * len(users), d["q"])


def _scores(r):
    return {"logprob": r.logprob, "entropy": r.entropy, "ids": r.top_ids, "alternatives": r.top_logprobs}


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


def _attention(q, k, v):
    """q [nq, hd] over k, v [L, nkv, hd] in fp32; zeros where there is no position."""
    nq, hd = q.shape
    nkv = k.shape[1]
    if not k.shape[0]:
        return torch.zeros_like(q)
    k, v = k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous()
    z = torch.matmul(k, q.float().view(nkv, nq // nkv, hd).transpose(1, 2).contiguous()) / math.sqrt(hd)
    p = torch.exp(z - z.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    return torch.matmul(p.transpose(1, 2).contiguous(), v).reshape(nq, hd).to(q.dtype)


def _logprobs(z, targets, top):
    """Log probabilities of fp32 logits z [rows, V]; -inf is masked, and a row with nothing left gives -inf and 0."""
    m = z.amax(-1, keepdim=True)
    some = m > -math.inf
    x = torch.where(some, z - torch.where(some, m, 0.0), z)
    e = torch.exp(x)
    sums = e.sum(-1, keepdim=True)
    log_sum = torch.where(some, torch.log(sums), 0.0)
    entropy = torch.where(some, log_sum - torch.where(e > 0, e * x, 0.0).sum(-1, keepdim=True) / torch.where(some, sums, 1.0), 0.0)
    d = {"logprob": x.gather(1, targets.long()[:, None])[:, 0] - log_sum[:, 0], "entropy": entropy[:, 0]}
    # the order of floats as integers, and the lower index first among equals
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (bits << 32) | (0xFFFFFFFF - torch.arange(z.shape[1], device=z.device))
    n = min(top, z.shape[1])
    ids = 0xFFFFFFFF - (torch.topk(key, n, dim=1).values & 0xFFFFFFFF)
    best = x.gather(1, ids) - log_sum
    d["ids"] = torch.where(best > -math.inf, ids, -1).to(torch.int32)
    d["alternatives"] = best
    return d if top else {**d, "ids": None, "alternatives": None}


def _run_plain(s):
    case, d = s.case, s.d
    kind = case["kind"]
    if kind == "head":
        x = d["hidden"].float()
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * d["gain"].float()
        return _logprobs(torch.matmul(x, d["lm_head"].float().t()), d["targets"], case["top"])
    if kind == "logits":
        return _logprobs(d["logits"], d["targets"], case["top"])
    if kind == "attend":
        return torch.stack([_attention(q, _value(k), _value(v)) for q, (k, v) in zip(d["q"], s.rows)])
    if kind == "cache":
        return [_value(_hold(t, "mxfp4")) for t in d["kv"][0]]
    if kind == "copy":
        if case["src"] == case["dst"]:
            return [[_value([t.clone() for t in held]) for held in layer] for layer in s.rows]
        return [[_value(_hold(_value(held), case["dst"])) for held in layer] for layer in s.rows]
    out = []
    for q, new in zip(d["q"], d["new"]):
        mine = [[torch.cat(parts) for parts in zip(held, _hold(t, case["cache"]))] for held, t in zip(s.rows[0], new)]
        out.append(_attention(q, _value(mine[0]), _value(mine[1])))
    return torch.stack(out)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- what a pass cannot do without


def _row_bytes(case, cache):
    """Bytes of one position's keys and values in a cache."""
    _, _, nkv, hd, _ = SHAPES[case["shape"]]
    return 2 * nkv * hd * (2 if cache == "f16" else 17 / 32)


def work(case):
    """Inputs, weights and cache read once, results written once; a multiply and an add per product."""
    kind = case["kind"]
    if kind in ("head", "logits"):
        rows = case["rows"]
        out = rows * (4 + 4 + 4 + case["top"] * 8)
        if kind == "logits":
            return {"bytes": rows * case["vocab"] * 4 + out, "flops": 4.0 * rows * case["vocab"]}
        hidden, _, _, _, vocab = SHAPES[case["shape"]]
        return {"bytes": 2 * vocab * hidden + rows * hidden * BYTES[case["io"]] + out,
                "flops": 2.0 * rows * vocab * hidden}
    _, nq, nkv, hd, _ = SHAPES[case["shape"]]
    if kind == "cache":
        return {"bytes": case["n"] * (2 * nkv * hd * (BYTES[case["io"]] + 4) + 2 * _row_bytes(case, "mxfp4")), "flops": 0}
    if kind == "copy":
        row = _row_bytes(case, case["src"]) + 2 * _row_bytes(case, case["dst"]) + 2 * nkv * hd * 4
        return {"bytes": LAYERS * case["n"] * row, "flops": 0}
    if kind == "attend":
        keys, read, rows = sum(_contexts(case)), sum(_contexts(case)), len(_contexts(case))
    else:  # the shared positions are read once
        rows = case["users"]
        keys, read = rows * (case["n"] + 1), case["n"] + rows
    return {"bytes": read * _row_bytes(case, case["cache"]) + 2 * rows * nq * hd * BYTES[case["io"]],
            "flops": 4.0 * nq * hd * keys}


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


def _softmax_of(q, k, v):
    nq, hd = q.shape
    group = nq // k.shape[1]
    out = torch.zeros((nq, hd), dtype=torch.float64, device=q.device)
    for h in range(nq):
        if k.shape[0]:
            z = (k[:, h // group] * q[h].double()).sum(-1) * hd ** -0.5
            out[h] = (torch.softmax(z, 0)[:, None] * v[:, h // group]).sum(0)
    return out


def exact(case, seed):
    d = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("head", "logits"):
        if kind == "head":
            x = d["hidden"].double()
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + float(torch.tensor(EPS, dtype=torch.float32)))
            z = torch.cat([(x * d["gain"].double()) @ w.double().t().contiguous() for w in d["lm_head"].split(16384)], -1)
        else:
            z = d["logits"].double()
        left = torch.isfinite(z).any(-1, keepdim=True)
        lp = torch.where(left, torch.log_softmax(torch.where(left, z, 0.0), -1), -math.inf)
        p = lp.exp()
        r = {"logprob": lp[torch.arange(len(lp)), d["targets"].long()],
             "entropy": -torch.where(p > 0, p * lp, 0.0).sum(-1), "ids": None, "alternatives": None}
        if case["top"]:
            best, at = torch.sort(lp, dim=-1, descending=True, stable=True)
            best, at = best[:, :case["top"]], at[:, :case["top"]]
            r["ids"], r["alternatives"] = torch.where(best > -math.inf, at, -1).to(torch.int32), best
        return r
    if kind == "cache":
        return [_nearest(t, "mxfp4") for t in d["kv"][0]]
    if kind == "copy":
        return [[_nearest(_nearest(t, case["src"]), case["dst"]) for t in layer] for layer in d["kv"]]
    held = [[_nearest(t, case["cache"]) for t in kv] for kv in d["kv"]]
    if kind == "attend":
        return torch.stack([_softmax_of(q, k, v) for q, (k, v) in zip(d["q"], held)])
    (k, v), out = held[0], []
    for q, new in zip(d["q"], d["new"]):
        nk, nv = (_nearest(t, case["cache"]) for t in new)
        out.append(_softmax_of(q, torch.cat([k, nk]), torch.cat([v, nv])))
    return torch.stack(out)
