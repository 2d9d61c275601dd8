"""Attention over caches of both types: given queries (kf_kv_attend), and decode and prefill on MXFP4 caches."""
import math

import numpy as np
import pytest

import synth
from oracle import stage_oracle as so
from tests import mx_ref
from tests.helpers import SeededModel, assert_hidden_close
from tests.test_gpu_cache import bare_stage, held, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


@pytest.fixture(scope="module")
def st():
    from paper_2609_34045_amd import stage
    return stage


def on(t, dtype=None):
    import torch
    x = torch.from_numpy(np.ascontiguousarray(t)).cuda()
    return x if dtype is None else x.to(dtype)


def want_of(q, k, v):
    """softmax(q K^T / sqrt(hd)) V in 64 bits for q [nq, hd], k, v [L, nkv, hd]; zeros without positions."""
    nq, hd = q.shape
    if not len(k):
        return np.zeros((nq, hd))
    return so.attention_rows(q[None].astype(np.float64), [k], [v], k.shape[1]).reshape(nq, hd)


def allowed(q, k, v, want, cache, eps):
    """How far a row's output may be off, [nq, 1].

    With scores s in log2 units and S the largest sum of |products| of a score, a score is off by the rounding of the
    query (two fp16 parts: 2^-22 of each value; one part over an fp16 cache: 2^-11) and of hd fp32 additions
    (2^-24 S each): ds.  A probability is off by ln 2 ds, 2^-22 for the exponential, and its own rounding (two bf16
    parts 2^-17, one fp16 part 2^-11).  Numerator and denominator each by that and 2^-24 for each of the additions along a
    chain (fewer than 200, the sums being split), relative to sum p |v|; the output's own rounding comes on top."""
    nq, hd = q.shape
    if not len(k):
        return np.zeros((nq, 1))
    kk = np.repeat(np.abs(k), nq // k.shape[1], axis=1)  # [L, nq, hd]
    S = np.einsum("hd,lhd->hl", np.abs(q.astype(np.float64)), kk).max(-1) * math.log2(math.e) / math.sqrt(hd)
    ds = S * ((2.0 ** -22 if cache == "mxfp4" else 2.0 ** -11) + hd * 2.0 ** -24)
    rel = math.log(2) * ds + 2.0 ** -22 + (2.0 ** -17 if cache == "mxfp4" else 2.0 ** -11) + 200 * 2.0 ** -24
    most = np.abs(v).max((0, 2))[np.arange(nq) // (nq // k.shape[1])]
    return (2 * rel * most + eps * np.abs(want).max(-1))[:, None] * 1.01


EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.mark.parametrize("cache", ["mxfp4", "f16"])
@pytest.mark.parametrize("io", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("hd,nkv,group,lens,paged", [
    (128, 2, 4, (200,), False), (64, 2, 4, (1, 64, 65, 0), True), (128, 1, 8, (3000, 63, 257), True),
    (64, 3, 1, (0,), False), (128, 2, 5, (127, 129), False), (64, 1, 8, (1500,), True), (128, 8, 1, (2, 700, 1100, 1024), False)])
def test_against_64_bits(torch, st, cache, io, hd, nkv, group, lens, paged):
    """Every length around pages and splits, rows without positions, group sizes and types, with other values in the
    cache behind each row's last position."""
    ctx = max(lens) + 100
    g = bare_stage(st, nkv, hd, layers=2, group=group)
    kv = g.kv(4, ctx, 4 * ((ctx + 63) // 64) if paged else None, dtype=cache)
    want, tol, q = [], [], on(rows(5, len(lens), nkv * group, hd, 1.5), getattr(torch, io))
    for b, n in enumerate(lens):
        k, v = rows(10 + b, ctx, nkv, hd, 2.0), rows(20 + b, ctx, nkv, hd)
        kv.write(1, 3 - b, 0, on(k), on(v))
        k, v = held(k, cache)[:n], held(v, cache)[:n]
        qb = q[b].float().cpu().numpy()
        want.append(want_of(qb, k, v))
        tol.append(allowed(qb, k, v, want[-1], cache, EPS[io]))
    got = kv.attend(1, [3 - b for b in range(len(lens))], lens, q)
    assert got.dtype == q.dtype and got.shape == q.shape
    err = np.abs(got.float().cpu().numpy().astype(np.float64) - np.stack(want))
    assert np.all(err <= np.stack(tol)), (err / np.maximum(np.stack(tol), 1e-300)).max()
    kv.attend(1, [3 - b for b in range(len(lens))], lens, q, out=q)  # in place
    assert torch.equal(q, got)
    g.sync()
    kv.close()
    g.close()


def test_long_rows_and_repeated_users(torch, st):
    """A context of several splits a row at several lengths of one user at once; the same bits on every call."""
    hd, nkv, group, n = 128, 2, 4, 20001
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(1, n, (n + 63) // 64, dtype="mxfp4")
    k, v = rows(1, n, nkv, hd, 1.3), rows(2, n, nkv, hd)
    kv.write(0, 0, 0, on(k), on(v))
    k, v = held(k, "mxfp4"), held(v, "mxfp4")
    q = on(rows(3, 4, nkv * group, hd))
    lens = [n, 4096, 5000, 1]
    got = kv.attend(0, [0] * 4, lens, q)
    for b, m in enumerate(lens):
        qb = q[b].cpu().numpy()
        w = want_of(qb, k[:m], v[:m])
        err = np.abs(got[b].cpu().numpy() - w)
        assert np.all(err <= allowed(qb, k[:m], v[:m], w, "mxfp4", EPS["float32"])), b
    assert torch.equal(kv.attend(0, [0] * 4, lens, q), got)
    one = kv.attend(0, [0], [1], q[3:].contiguous())  # alone, from one split
    assert torch.allclose(one, got[3:], rtol=1e-5, atol=1e-6)
    g.sync()
    kv.close()
    g.close()


def test_the_longest_cache(torch, st):
    """1,048,576 positions of four users, a cache of more than 2^32 bytes: the last user's last and middle positions are
    written, read, attended to, forked and copied into a cache of the other type."""
    hd, nkv, group, n = 128, 8, 2, 1 << 20
    g = bare_stage(st, nkv, hd, group=group)
    kv, half = g.kv(4, n, dtype="mxfp4"), g.kv(1, n)
    assert kv.format()[1] > 1 << 32
    at = [(500_003, 70), (n - 130, 130)]
    parts = [(rows(2 * i, m, nkv, hd), rows(2 * i + 1, m, nkv, hd, 1e3)) for i, (_, m) in enumerate(at)]
    for (p, m), (k, v) in zip(at, parts):
        kv.write(0, 3, p, on(k), on(v))
    kv.set_len(3, n)
    parts = [(held(k, "mxfp4"), held(v, "mxfp4")) for k, v in parts]
    # the other positions' keys and values are zero: score 0 each, and nothing added
    k, v = (np.concatenate([parts[0][i], parts[1][i], np.zeros((1, nkv, hd))]) for i in (0, 1))
    count = np.r_[np.ones(200), n - 200]
    q = rows(9, 1, nkv * group, hd, 2.0)
    s = np.einsum("hd,lhd->hl", q[0].astype(np.float64), np.repeat(k, group, axis=1)) / math.sqrt(hd)
    w = count * np.exp(s - s.max(1, keepdims=True))
    want = np.einsum("hl,lhd->hd", w, np.repeat(v, group, axis=1)) / w.sum(1, keepdims=True)
    # `allowed` of the part of the probability that these keys have, and the longer sums: 16 positions of up to 16 pages in a
    # lane, up to 1024 splits by four waves, 400 additions more than it counts
    part = (w[:, :-1].sum(1) / w.sum(1))[:, None]
    tol = (allowed(q[0], k, v, want, "mxfp4", 0) + 2 * 400 * 2.0 ** -24 * np.abs(v).max()) * part + 2.0 ** -24 * np.abs(want).max()
    assert tol.max() < 0.01 * np.abs(want).max()
    kv.fork(3, 0)
    half.copy(kv, 3, 0, 0, n)
    for cache, user in ((kv, 3), (kv, 0), (half, 0)):
        for (p, m), (pk, pv) in zip(at, parts):
            for got, x in zip(cache.read(0, user, p - 1 if p + m < n else p, m + (p + m < n)), (pk, pv)):
                got = got.cpu().numpy()
                assert np.array_equal(got[-m:], x) and not got[:-m].any()
    for user in (3, 0):
        got = kv.attend(0, [user], [n], on(q))[0].cpu().numpy()
        assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()
    g.sync()
    kv.close()
    half.close()
    g.close()


@pytest.mark.parametrize("scale_q,scale_k", [(1e-6, 1.0), (1e4, 1e-4), (1.0, 200.0), (3e-30, 1e3), (1e5, 1e4)])
def test_queries_and_keys_of_any_size(torch, st, scale_q, scale_k):
    """Tiny and large queries keep their bits, a sharply peaked row finds its key, and values near both ends of the
    format come out in proportion."""
    hd = 64
    g = bare_stage(st, 1, hd, group=8)
    kv = g.kv(1, 300, dtype="mxfp4")
    k, v = rows(1, 300, 1, hd, scale_k), rows(2, 300, 1, hd, 1e-5)
    v[:, :, 32:] *= 1e9
    kv.write(0, 0, 0, on(k), on(v))
    k, v = held(k, "mxfp4"), held(v, "mxfp4")
    q = rows(3, 1, 8, hd, scale_q)
    got = kv.attend(0, [0], [300], on(q))[0].cpu().numpy()
    w = want_of(q[0], k, v)
    for part in (slice(0, 32), slice(32, 64)):  # each block of values by its own size
        err = np.abs(got[:, part] - w[:, part])
        assert np.all(err <= allowed(q[0], k, v[:, :, part], w[:, part], "mxfp4", EPS["float32"]))
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("io", ["float32", "bfloat16"])
@pytest.mark.parametrize("power", [110, 113, 117, 121])
def test_queries_near_the_top_of_the_range(torch, st, io, power):
    """Queries whose scores with small keys are finite find the key of the largest score: every other probability is
    2^-(a huge number), so that the row is that key's value to the last bit."""
    hd, n = 64, 300
    g = bare_stage(st, 1, hd, group=8)
    kv = g.kv(1, n, dtype="mxfp4")
    k, v = rows(1, n, 1, hd, 1e-5), rows(2, n, 1, hd)
    kv.write(0, 0, 0, on(k), on(v))
    k, v = held(k, "mxfp4"), held(v, "mxfp4")
    q = on(rows(3, 1, 8, hd) * np.float32(2.0 ** power), getattr(torch, io))
    s = q[0].float().cpu().numpy().astype(np.float64) @ k[:, 0].T
    order = np.sort(s, axis=1)
    size = np.abs(q[0].float().cpu().numpy().astype(np.float64)) @ np.abs(k[:, 0]).T
    assert np.all(order[:, -1] - order[:, -2] > 2.0 ** -16 * size.max(1))  # above what 22-bit queries and fp32 sums lose
    got = kv.attend(0, [0], [n], q)[0].float().cpu().numpy()
    assert np.array_equal(got, on(v[s.argmax(1), 0].astype(np.float32), getattr(torch, io)).float().cpu().numpy())
    g.sync()
    kv.close()
    g.close()


def test_a_peak_beside_a_long_flat_tail(torch, st):
    """One key of probability near a half and 8000 that share the rest, each far below it: they count to the last bit."""
    hd, n = 64, 8001
    g = bare_stage(st, 1, hd, group=1)
    kv = g.kv(1, n, dtype="mxfp4")
    k = np.zeros((n, 1, hd), np.float32)
    k[:, 0, 0] = 1.0
    k[4000, 0, 0] = 6.0
    v = rows(2, n, 1, hd)
    v[4000] = 0
    kv.write(0, 0, 0, on(k), on(v))
    q = np.zeros((1, 1, hd), np.float32)
    q[0, 0, 0] = math.log(8000) / 5 * math.sqrt(hd)
    v = held(v, "mxfp4")
    got = kv.attend(0, [0], [n], on(q))[0, 0].cpu().numpy()
    w = want_of(q[0], held(k, "mxfp4"), v)[0]
    # The tail's keys have one score and so one error: ln 8000 2^-22 of the query's parts, 13 2^-24 of the exponential's
    # argument, 2^-23 of itself, 2^-22 of its parts, together below 2^-18 of the tail's sum; the fp32 sums of at most 64
    # steps in a row, each off by 2^-24 of partial sums of the size of `tail`, stay below 2^-18 of that.
    tail = np.sqrt((np.delete(v[:, 0], 4000, 0) ** 2).sum(0)) / 16000
    assert np.all(np.abs(got - w) <= 2.0 ** -17 * (np.abs(w) + tail))
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["mxfp4", "f16"])
def test_a_nan_query_gives_nan_in_its_head_only(torch, st, cache):
    g = bare_stage(st, 1, 64, group=4)
    kv = g.kv(1, 700, dtype=cache)
    kv.write(0, 0, 0, on(rows(1, 700, 1, 64)), on(rows(2, 700, 1, 64)))
    q = on(rows(3, 2, 4, 64))
    clean = kv.attend(0, [0, 0], [700, 10], q)
    q[0, 2, 7] = float("nan")
    got = kv.attend(0, [0, 0], [700, 10], q)
    bad = torch.zeros(2, 4, dtype=torch.bool, device="cuda")
    bad[0, 2] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])
    kv.close()
    g.close()


def test_refusals(torch, st):
    g = bare_stage(st, 1, 64, layers=2, group=2)
    kv = g.kv(2, 100, 3, dtype="mxfp4")
    kv.write(0, 0, 0, on(rows(1, 64, 1, 64)), on(rows(2, 64, 1, 64)))
    q = on(rows(3, 1, 2, 64))

    def refused(status, *args, **kw):
        with pytest.raises(st.KFError) as e:
            kv.attend(*args, **kw)
        assert e.value.status == status
    refused(3, 0, [0], [65], q)       # on no page of the user's
    refused(3, 0, [0], [101], q)
    refused(3, 0, [1], [1], q)
    refused(1, 0, [0], [-1], q)
    refused(1, 0, [2], [1], q)
    refused(1, 2, [0], [1], q)        # no such layer
    refused(1, 0, [0] * 5, [1] * 5, on(rows(3, 5, 2, 64)))
    refused(1, 0, [], [], on(rows(3, 1, 2, 64))[:0])
    odd = torch.zeros(129, device="cuda")[1:].view(1, 2, 64)
    refused(1, 0, [0], [1], odd)
    with pytest.raises(ValueError):
        kv.attend(0, [0], [1], on(rows(3, 1, 2, 32)))
    with pytest.raises(TypeError):
        kv.attend(0, [0], [1], q.double())
    kv.attend(0, [1], [0], q)         # a user without pages, and nothing to attend
    g.sync()
    kv.close()
    g.close()


def test_captured_and_replayed_on_another_stream(torch, st):
    """A captured call reads what the cache holds at each replay, among eager calls that use the same workspace."""
    hd, nkv, group, n = 128, 2, 4, 3000
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(2, n, dtype="mxfp4")
    kvs = [[on(rows(10 * i + j, n, nkv, hd)) for j in range(2)] for i in range(3)]
    kv.write(0, 0, 0, *kvs[0])
    kv.write(0, 1, 0, *kvs[1])
    q = on(rows(3, 1, nkv * group, hd))
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)
    with torch.cuda.stream(side):
        eager = [kv.attend(0, [u], [n], q).clone() for u in (0, 1)]
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            kv.attend(0, [0], [n], q, out=out)
        for _ in range(3):
            graph.replay()
            side.synchronize()
            assert torch.equal(out, eager[0])
            assert torch.equal(kv.attend(0, [1], [n], q), eager[1])
        kv.write(0, 0, 0, *kvs[2])
        after = kv.attend(0, [0], [n], q).clone()
        graph.replay()
        side.synchronize()
    assert torch.equal(out, after) and not torch.equal(after, eager[0])
    g.sync()
    kv.close()
    g.close()


# ---------------------------------------------------------------- decode and prefill


def layer_with(x, w, shape, layer, users, positions, kv):
    """One decoder layer in 64 bits whose attention reads the keys and values that the cache holds, and the keys and
    values that it would append."""
    n, nq, nkv, hd = len(x), shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    xn = so.rms_norm(x, w["attn_norm"], shape.rms_eps)
    q, k, v = ((xn @ w[name].T).reshape(n, -1, hd) for name in ("wq", "wk", "wv"))
    if shape.qk_norm:
        q, k = so.rms_norm(q, w["q_norm"], shape.rms_eps), so.rms_norm(k, w["k_norm"], shape.rms_eps)
    pos = np.asarray(positions)
    q, k = so.rope(q, pos, shape.rope_theta), so.rope(k, pos, shape.rope_theta)
    read = {u: [t.cpu().numpy().astype(np.float64) for t in kv.read(layer, u, 0, int(pos[[a == u for a in users]].max()) + 1)]
            for u in set(users)}
    o = so.attention_rows(q, [read[u][0][:p + 1] for u, p in zip(users, pos)],
                          [read[u][1][:p + 1] for u, p in zip(users, pos)], nkv)
    x = x + o @ w["wo"].T
    new = [(read[u][0][p], read[u][1][p]) for u, p in zip(users, pos)]
    return x + so.mlp_swiglu(so.rms_norm(x, w["mlp_norm"], shape.rms_eps), w["wg"], w["wu"], w["wd"]), k, v, new


def check_step(x, got, model, shape, layers, users, positions, kv, what):
    """The hidden rows of a step, and that what it appended are the roundings of the keys and values: the same element in
    nearly all places.  Where a value lies next to the middle of two elements (or a block's largest next to the border of
    two exponents) the two roundings differ by at most one step, 2 units of the block's power of two, while its largest
    element is 4 units or more: never by more than half of that element."""
    x = np.asarray(x, np.float64)
    for l in range(layers):
        w = {k: so.bf16_to_f64(v) for k, v in model.layer(l).items()}
        x, k, v, new = layer_with(x, w, shape, l, users, positions, kv)
        for mine, theirs in ((k, [n[0] for n in new]), (v, [n[1] for n in new])):
            want, theirs = mx_ref.stored(mine), np.stack(theirs)
            top = np.abs(want.reshape(-1, 32)).max(-1, keepdims=True)
            off = np.abs(want - theirs).reshape(-1, 32)
            assert np.mean(off > 0) < 0.03 and np.all(off <= top * 0.5), (what, l, np.mean(off > 0))
    assert_hidden_close(got.float().cpu().numpy(), x, what=what)


@pytest.mark.parametrize("shape", [synth.SHAPE_TINY, synth.SHAPE_QWEN3_TINY,
                                   synth.ModelShape(2, 512, 8, 2, 128, 704, 0, qk_norm=True)], ids=["tiny", "qwen3", "hd128"])
@pytest.mark.parametrize("paged,ordered", [(False, False), (True, True)])
def test_prefill_and_decode_on_a_4bit_cache(torch, st, shape, paged, ordered):
    layers, cfg = 2, 61
    model = SeededModel(shape, cfg)
    g = st.Stage(shape, 0, layers, model.layer)
    if ordered:
        g.set_flags(st.KF_STAGE_ORDERED)
    kv = g.kv(3, 300, 12 if paged else None, dtype="mxfp4")
    pos = 0
    for i, n in enumerate((70, 1, 100)):
        h = synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, i, n, shape.hidden)
        y = g.prefill(kv, 1, pos, hidden=on(h), noalloc=i == 2)
        check_step(h, y, model, shape, layers, [1] * n, list(range(pos, pos + n)), kv, f"prefill {n} at {pos}")
        pos += n
    h = synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, 9, 5, shape.hidden)
    g.prefill(kv, 0, 0, hidden=on(h))
    for step, users in enumerate(([1], [1, 0], [2, 0, 1], [1], [2])):
        x = synth.hidden_states(cfg, synth.STREAM_DECODE_HIDDEN, step, len(users), shape.hidden)
        at = [kv.len(u) for u in users]
        y = g.decode(kv, users, at, hidden=on(x))
        check_step(x, y, model, shape, layers, users, at, kv, f"decode {step}")
    g.sync()
    kv.close()
    g.close()


def test_decode_appends_what_a_write_would(torch, st):
    """The first layer's new keys and values do not depend on the cache: on an MXFP4 cache they are the roundings of
    those on an fp16 cache."""
    for shape in (synth.SHAPE_TINY, synth.SHAPE_QWEN3_TINY):
        model = SeededModel(shape, 62)
        g = st.Stage(shape, 0, 1, model.layer)
        a, b = g.kv(4, 100), g.kv(4, 100, dtype="mxfp4")
        x = on(synth.hidden_states(62, synth.STREAM_DECODE_HIDDEN, 0, 4, shape.hidden))
        for kv in (a, b):
            for step in range(2):
                for batch in ([0], [1, 2, 3]):
                    g.decode(kv, batch, [step] * len(batch), hidden=x[:len(batch)].contiguous())
        for u in range(4):
            for t, w in zip(b.read(0, u, 0, 2), a.read(0, u, 0, 2)):
                assert np.array_equal(t.cpu().numpy(), mx_ref.stored(w.cpu().numpy())), u
        g.sync()
        a.close()
        b.close()
        g.close()


@pytest.mark.parametrize("cache", ["mxfp4", "f16"])
def test_forked_users_decode_together(torch, st, cache):
    """Users that share a prompt's pages step together like users with copies of their own, and the ring's rule that a
    step finds its pages or changes nothing holds for copies too."""
    shape = synth.SHAPE_TINY
    model = SeededModel(shape, 63)
    g = st.Stage(shape, 0, 2, model.layer)
    shared, apart = g.kv(4, 200, 6, dtype=cache), g.kv(4, 200, dtype=cache)
    h = on(synth.hidden_states(63, synth.STREAM_PREFILL_HIDDEN, 0, 70, shape.hidden))
    g.prefill(shared, 0, 0, hidden=h)
    g.prefill(apart, 0, 0, hidden=h)
    for u in (1, 2, 3):
        shared.fork(0, u)
        apart.fork(0, u)
    assert shared.pages() == (6, 4)
    for step in range(3):
        x = on(synth.hidden_states(63, synth.STREAM_DECODE_HIDDEN, step, 4, shape.hidden))
        y, z = (g.decode(kv, [0, 1, 2, 3], [70 + step] * 4, hidden=x) for kv in (shared, apart))
        assert torch.equal(y, z), step
        assert shared.pages() == (6, 1)  # three copies of the last page, the fourth user writes in place
    shared.fork(1, 0)
    shared.fork(1, 2)
    shared.fork(1, 3, 72)
    assert shared.pages() == (6, 4)
    shared.fork(1, 2, 64)
    x = on(synth.hidden_states(63, synth.STREAM_DECODE_HIDDEN, 5, 3, shape.hidden))
    apart.fork(1, 0)
    apart.fork(1, 3, 72)
    y, z = (g.decode(kv, [3, 1, 0], [72, 73, 73], hidden=x) for kv in (shared, apart))
    assert torch.equal(y, z) and shared.pages() == (6, 2)
    g.sync()
    shared.close()
    apart.close()
    g.close()


def test_a_ring_counts_copies_of_shared_pages(torch, st):
    """A ring's members admit a call only if their pools hold the copies that shared pages need, and forked users on
    4-bit caches then generate what users with prompts of their own do."""
    from paper_2609_34045_amd.ring import Ring
    shape = synth.SHAPE_TINY
    model = SeededModel(shape, 64)
    stages = [st.Stage(shape, 0, 1, model.layer, model.head()), st.Stage(shape, 1, 2, model.layer)]
    prompt = on(synth.tokens(64, 0, 70, shape.vocab))

    def ring_of(pages):
        caches = [s.kv(3, 192, pages, dtype="mxfp4") for s in stages]
        return caches, Ring(stages, caches, 2, 128)

    caches, ring = ring_of(4)
    first = ring.prefill(0, prompt)
    for kv in caches:
        kv.fork(0, 1)
        kv.fork(0, 2)
    assert caches[0].pages() == (4, 2)
    last = first.repeat(3)
    caches[1].write(1, 2, 128, *(torch.zeros(1, 2, 64, device="cuda") for _ in range(2)))  # takes a page: one left in member 1
    before = [(kv.pages(), [kv.len(u) for u in range(3)]) for kv in caches]
    with pytest.raises(st.KFError) as e:
        ring.generate([[0, 1, 2]], last, 2)
    assert e.value.status == 2 and "member 1" in e.value.message
    assert before == [(kv.pages(), [kv.len(u) for u in range(3)]) for kv in caches]
    caches[1].set_len(2, 70)
    got = ring.generate([[0, 1, 2]], last, 3).cpu().numpy()
    assert caches[0].pages() == (4, 0)
    ring.close()
    for kv in caches:
        kv.close()
    caches, ring = ring_of(9)
    for u in range(3):
        assert torch.equal(ring.prefill(u, prompt), first)
    assert np.array_equal(ring.generate([[0, 1, 2]], last, 3).cpu().numpy(), got)
    ring.close()
    for kv in caches:
        kv.close()
    for s in stages:
        s.sync()
        s.close()
