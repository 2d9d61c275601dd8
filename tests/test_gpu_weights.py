"""Attention weights of cached positions (kf_kv_track, kf_kv_weigh) and eviction by them (kf_kv_evict)."""
import math

import numpy as np
import pytest

import synth
from oracle import stage_oracle as so
from tests.helpers import SeededModel
from tests.test_gpu_attend import on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_cache import bare_stage, check, held, rows
from tests.test_gpu_tree import draft, want_of

pytestmark = pytest.mark.gpu


def weight_of(q, k, length):
    """What query row q [nq, hd] adds to each of k [L, nkv, hd]'s positions, [nkv, L], and how far that may be off.

    With scores in log2 units and S the largest sum of |products|: a score is off by the query's rounding (two fp16 parts,
    2^-22, or none) and hd + 4 fp32 roundings (2^-24 S each), and so is the logarithm of the sum of the 2^s, which takes
    fewer than 400 additions along a chain besides; ln 2 of the two makes a probability's relative error, with 2^-22 for each of
    the exponentials and 2^-20 for the logarithm (2^-24 of up to 16)."""
    nq, hd = q.shape
    nkv = k.shape[1]
    w, tol = np.zeros((nkv, len(k))), np.zeros((nkv, len(k)))
    for h in range(nq if length else 0):
        g = h // (nq // nkv)
        s = k[:length, g] @ q[h].astype(np.float64) / math.sqrt(hd)
        p = np.exp(s - s.max())
        p /= p.sum()
        S = (np.abs(k[:length, g]) @ np.abs(q[h].astype(np.float64))).max() * math.log2(math.e) / math.sqrt(hd)
        ds = S * (2.0 ** -22 + (hd + 4) * 2.0 ** -24)
        w[g, :length] += p
        tol[g, :length] += p * (2 * math.log(2) * ds + 400 * 2.0 ** -24 + 2 * 2.0 ** -22 + 2.0 ** -20)
    return w, tol


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("io", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("hd,nkv,group,at,paged", [
    # (user, positions) of each row
    (128, 2, 4, [(0, 200)], False), (64, 2, 4, [(3, 1), (1, 64), (0, 65), (2, 0)], True),
    (128, 1, 8, [(1, 3000 - 31 + i) for i in range(32)], True), (64, 3, 1, [(0, 0)], False),
    (128, 2, 5, [(1, 127), (0, 129), (1, 5), (1, 127), (0, 64)], False), (64, 1, 7, [(2, 1500 + i) for i in range(9)], True),
    (128, 8, 1, [(u, 2 + 300 * u + i) for i in range(7) for u in range(4)], False)])
def test_weights_against_64_bits(torch, st, cache, io, hd, nkv, group, at, paged):
    """One and many rows of one and several users in any order, added to what is there; other users, layers and positions
    past a user's last are left as they are, and the same call gives the same bits."""
    ctx = max(n for _, n in at) + 100
    g = bare_stage(st, nkv, hd, layers=2, group=group)
    kv = g.kv(4, ctx, 4 * ((ctx + 63) // 64) if paged else None, dtype=cache)
    kv.track()
    q = on(rows(5, len(at), nkv * group, hd, 1.5), getattr(torch, io))
    want, tol = [], []
    for u in range(4):
        k, v = rows(10 + u, ctx, nkv, hd, 2.0), rows(20 + u, ctx, nkv, hd)
        kv.write(1, u, 0, on(k), on(v))
        old = np.random.default_rng(u).uniform(0, 1, (nkv, ctx)).astype(np.float32)
        kv.set_weights(1, u, 0, on(old))
        w, t = old.astype(np.float64), np.zeros((nkv, ctx))
        for b, (user, n) in enumerate(at):
            if user == u:
                a, e = weight_of(q[b].float().cpu().numpy(), held(k, cache), n)
                w, t = w + a, t + e
        want.append(w)
        tol.append(t + np.where(t > 0, 2.0 ** -24 * 300 * w, 0))
    for _ in range(2):
        kv.weigh(1, [u for u, _ in at], [n for _, n in at], q)
        got = [kv.weights(1, u, 0, ctx).cpu().numpy() for u in range(4)]
        for u in range(4):
            assert np.all(np.abs(got[u] - want[u]) <= tol[u] * 1.01), (u, np.max(np.abs(got[u] - want[u]) / np.maximum(tol[u], 1e-30)))
            assert not kv.weights(0, u, 0, ctx).any()
            old = np.random.default_rng(u).uniform(0, 1, (nkv, ctx)).astype(np.float32)
            kv.set_weights(1, u, 0, on(old))
        if _ == 0:
            first = got
    assert all(np.array_equal(a, b) for a, b in zip(first, got))
    g.sync()
    kv.close()
    g.close()


def test_a_long_cache_and_a_flat_tail(torch, st):
    """2^20 positions of two users, past 2^32 bytes: the sum of what is added is the number of heads, small weights keep their bits."""
    hd, nkv, group, n = 128, 8, 2, 1 << 20
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(2, n)
    kv.track()
    k = rows(1, 300, nkv, hd, 1.5)
    kv.write(0, 1, n - 300, on(k), on(k))
    q = rows(3, 1, nkv * group, hd, 2.0)
    kv.weigh(0, [1], [n], on(q))
    got = kv.weights(0, 1, 0, n).double().cpu().numpy()
    w = np.zeros((nkv, n))
    for h in range(nkv * group):
        s = np.zeros(n)
        s[n - 300:] = held(k, "f16")[:, h // group] @ q[0, h].astype(np.float64) / math.sqrt(hd)
        p = np.exp(s - s.max())
        w[h // group] += p / p.sum()
    # `weight_of`, with scores of up to 40 in log2 units here and a chain of up to 2^20 / 64 additions at the most
    assert np.all(np.abs(got - w) <= w * (2 * math.log(2) * 40 * (2.0 ** -22 + 132 * 2.0 ** -24) + 2.0 ** -10))
    assert np.all(np.abs(got.sum(1) - group) <= group * 2.0 ** -10)
    assert not kv.weights(0, 0, 0, n).any()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_queries_that_are_not_finite_add_nothing(torch, st, cache):
    g = bare_stage(st, 2, 64, group=4)
    kv = g.kv(1, 700, dtype=cache)
    kv.track()
    kv.write(0, 0, 0, on(rows(1, 700, 2, 64)), on(rows(2, 700, 2, 64)))
    q = on(rows(3, 3, 8, 64))
    alone = []
    for h in range(8):
        x = torch.full_like(q, math.nan)
        x[:, h] = q[:, h]
        kv.set_weights(0, 0, 0, torch.zeros((2, 700), device="cuda"))
        kv.weigh(0, [0] * 3, [700, 10, 300], x)
        alone.append(kv.weights(0, 0, 0, 700).clone())
        assert torch.isfinite(alone[-1]).all() and not alone[-1][1 - h // 4].any()
    kv.set_weights(0, 0, 0, torch.zeros((2, 700), device="cuda"))
    kv.weigh(0, [0] * 3, [700, 10, 300], q)
    assert torch.allclose(kv.weights(0, 0, 0, 700), sum(alone), rtol=2.0 ** -20, atol=0)
    x = q.clone()
    x[0, 1, 3], x[2, 6, 7] = math.inf, -math.inf
    kv.set_weights(0, 0, 0, torch.zeros((2, 700), device="cuda"))
    kv.weigh(0, [0] * 3, [700, 10, 300], x)
    w = kv.weights(0, 0, 0, 700)
    assert torch.isfinite(w).all() and abs(w[0].sum().item() - 11) < 1e-3 and abs(w[1].sum().item() - 11) < 1e-3
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("shape", [synth.ModelShape(1, 512, 8, 2, 64, 1408, 1000), synth.ModelShape(1, 384, 8, 2, 64, 1024, 1000, qk_norm=True),
                                   synth.ModelShape(1, 512, 8, 2, 128, 704, 0, qk_norm=True)], ids=["tiny", "qwen3", "hd128"])
def test_prefill_and_decode_steps_add_theirs(torch, st, cache, shape):
    """The window's tokens of each chunk and every row of a step, over what the cache holds; new positions start at zero,
    whatever weight lay there."""
    cfg, window = 71, 12
    model = SeededModel(shape, cfg)
    w = {k: so.bf16_to_f64(v) for k, v in model.layer(0).items()}
    g = st.Stage(shape, 0, 1, model.layer)
    kv = g.kv(3, 300, 12, dtype=cache)
    kv.track(window)
    want, tol = np.zeros((3, shape.n_kv_heads, 300)), np.zeros((3, shape.n_kv_heads, 300))
    for u in range(3):
        kv.set_weights(0, u, 0, torch.full((shape.n_kv_heads, 300), 5.0, device="cuda"))

    def add(x, users, positions, tokens):
        """Row i at positions[i]; rows from `tokens` on count."""
        xn = so.rms_norm(np.asarray(x, np.float64), w["attn_norm"], shape.rms_eps)
        q = (xn @ w["wq"].T).reshape(len(x), -1, shape.head_dim)
        if shape.qk_norm:
            q = so.rms_norm(q, w["q_norm"], shape.rms_eps)
        q = so.rope(q, np.asarray(positions), shape.rope_theta)
        for i in range(len(x)):
            want[users[i], :, positions[i]] = tol[users[i], :, positions[i]] = 0
        for i in range(tokens, len(x)):
            n = positions[i] + 1
            k = kv.read(0, users[i], 0, n)[0].double().cpu().numpy()
            a, e = weight_of(q[i], k, n)
            # the queries' inputs and they themselves are held in fp16 (2^-11 each): a score of sum of |products| S is off
            # by 2 2^-11 S, which moves a probability by that and the sum's like it
            nq, nkv = shape.n_q_heads, shape.n_kv_heads
            S = max((np.abs(k[:, h // (nq // nkv)]) @ np.abs(q[i, h])).max() for h in range(nq)) / math.sqrt(shape.head_dim)
            want[users[i], :, :n] += a
            tol[users[i], :, :n] += e + a * math.expm1(2 * 2 * 2.0 ** -11 * S)

    def compare(what):
        for u in range(3):
            n = kv.len(u)
            if n:
                got = kv.weights(0, u, 0, n).double().cpu().numpy()
                assert np.all(np.abs(got - want[u, :, :n]) <= tol[u, :, :n] * 1.01 + 1e-7), (what, u)
    pos = 0
    for i, n in enumerate((70, 1, 100, 12)):
        h = synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, i, n, shape.hidden)
        g.prefill(kv, 1, pos, hidden=on(h), noalloc=i == 2)
        add(h, [1] * n, list(range(pos, pos + n)), max(n - window, 0))
        pos += n
        compare(f"chunk {i}")
    kv.track(0)
    h = synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, 9, 5, shape.hidden)
    g.prefill(kv, 0, 0, hidden=on(h))
    add(h, [0] * 5, list(range(5)), 5)
    compare("no window")
    for step, users in enumerate(([1], [1, 0], [2, 0, 1], [1], [2])):
        x = synth.hidden_states(cfg, synth.STREAM_DECODE_HIDDEN, step, len(users), shape.hidden)
        at = [kv.len(u) for u in users]
        g.decode(kv, users, at, hidden=on(x))
        add(x, users, at, 0)
        compare(f"decode {step}")
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("ordered", [False, True])
def test_tracking_leaves_what_a_stage_computes(torch, st, cache, ordered):
    """Prefill and decode steps on a tracked cache give the bits that they give on another (batch 1 in a fixed order)."""
    shape = synth.SHAPE_TINY
    model = SeededModel(shape, 72)
    g = st.Stage(shape, 0, 2, model.layer)
    g.set_flags(st.KF_STAGE_ORDERED if ordered else 0)
    kvs = [g.kv(2, 300, dtype=cache) for _ in range(2)]
    kvs[1].track(8)
    outs = []
    for kv in kvs:
        y = [g.prefill(kv, u, 0, hidden=on(synth.hidden_states(72, synth.STREAM_PREFILL_HIDDEN, u, 80, shape.hidden))) for u in range(2)]
        for step in range(4):
            users = [0, 1] if step % 2 or not ordered else [0]
            x = on(synth.hidden_states(72, synth.STREAM_DECODE_HIDDEN, step, len(users), shape.hidden))
            y.append(g.decode(kv, users, [kv.len(u) for u in users], hidden=x))
        outs.append([t.clone() for t in y])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for kv in kvs:
        kv.close()
    g.close()


def test_weights_go_with_their_positions(torch, st):
    """Written positions start at zero, copies and forks bring theirs (zero from an untracked cache), accepted positions
    move with theirs."""
    g = bare_stage(st, 2, 64, layers=2)
    a, b, plain = g.kv(3, 200, 12), g.kv(1, 300, dtype="mxfp4"), g.kv(1, 200)
    a.track()
    b.track()
    assert a.format()[1] >= g.kv(3, 200, 12).format()[1] + 2 * 2 * 200 * 4 * 4  # weights of three users, and what one keeps
    x = [on(rows(i, 150, 2, 64)) for i in range(2)]
    for l in range(2):
        a.write(l, 0, 0, *x)
        plain.write(l, 0, 0, *x)
    a.set_len(0, 150)
    w = [torch.rand((2, 150), device="cuda") for _ in range(2)]
    for l in range(2):
        a.set_weights(l, 0, 0, w[l])
    a.write(1, 0, 30, *(t[:10].contiguous() for t in x))
    w[1][:, 30:40] = 0
    a.fork(0, 1)
    a.fork(0, 2, 100)
    b.copy(a, 0, 0, 20, 100)
    for l in range(2):
        assert torch.equal(a.weights(l, 0, 0, 150), w[l]) and torch.equal(a.weights(l, 1, 0, 150), w[l])
        assert torch.equal(a.weights(l, 2, 0, 100), w[l][:, :100]) and not a.weights(l, 2, 100, 100).any()
        assert torch.equal(b.weights(l, 0, 20, 100), w[l][:, 20:120]) and not b.weights(l, 0, 0, 20).any()
    a.accept(1, 100, [3, 4, 40])
    at = list(range(100)) + [103, 104, 140]
    for l in range(2):
        assert torch.equal(a.weights(l, 1, 0, 103), w[l][:, at]) and torch.equal(a.weights(l, 0, 0, 150), w[l])
    a.copy(plain, 0, 2, 10, 50)
    for l in range(2):
        assert not a.weights(l, 2, 10, 50).any() and torch.equal(a.weights(l, 2, 60, 40), w[l][:, 60:100])
    for kv in (a, b, plain):
        kv.close()


def kept_of(w, keep, first, last):
    """The positions kept of weights w [n], by sorting."""
    n = len(w)
    order = sorted(range(first, n - last), key=lambda t: (math.isnan(w[t]), -w[t] if not math.isnan(w[t]) else 0, t))
    return sorted(list(range(first)) + order[:keep - first - last] + list(range(n - last, n)))


def evicted(kv, st_layers, nkv, cache, data, w, src, dst, keep, first, last, kept):
    """Checks what an eviction left of data[layer] = (k, v) and weights w[layer] [nkv, n]."""
    n = w[0].shape[1]
    assert kv.len(dst) == keep
    for l in range(st_layers):
        at = np.array([kept_of(w[l][g].tolist(), keep, first, last) for g in range(nkv)], dtype=np.int64)
        assert np.array_equal(kept[l].cpu().numpy(), at), l
        pick = lambda x: np.stack([held(x, cache)[at[g], g] for g in range(nkv)], 1)  # noqa: E731
        check(kv, l, dst, 0, *(pick(x) for x in data[l]), what=f"layer {l}")
        got = kv.weights(l, dst, 0, keep).cpu().numpy()
        assert np.array_equal(got, np.stack([w[l][g][at[g]] for g in range(nkv)]), equal_nan=True)
        if src != dst:
            check(kv, l, src, 0, *(held(x, cache)[:n] for x in data[l]), what="source")
            assert np.array_equal(kv.weights(l, src, 0, n).cpu().numpy(), w[l], equal_nan=True)


def some_weights(seed, nkv, n):
    """Weights over several magnitudes with zeros, equal ones and numbers that no attention gives."""
    r = np.random.default_rng(seed)
    w = np.exp(r.normal(size=(nkv, n)) * 3).astype(np.float32)
    w[r.uniform(size=w.shape) < 0.2] = 0
    w[:, ::3] = np.float32(2.0) ** np.round(np.log2(w[:, ::3] + 1e-6))
    if n > 20:
        w[0, 3], w[0, 7], w[-1, 11], w[-1, 12], w[0, 13], w[0, 14] = np.nan, -0.0, np.inf, -1.0, -np.inf, -np.nan
    return w


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("hd,nkv,n,keep,first,last,paged", [
    (64, 2, 300, 200, 4, 64, False), (128, 3, 300, 77, 0, 0, True), (128, 1, 1, 1, 0, 0, False), (64, 1, 65, 64, 64, 0, True),
    (64, 2, 130, 130, 3, 3, True), (128, 2, 1500, 1, 0, 1, False), (64, 3, 700, 0, 0, 0, True), (128, 2, 2100, 1999, 100, 900, True),
    (64, 1, 129, 66, 33, 33, False), (128, 1, 70, 69, 0, 69, True)])
def test_the_heaviest_stay(torch, st, cache, in_place, hd, nkv, n, keep, first, last, paged):
    g = bare_stage(st, nkv, hd, layers=3)
    ctx = n + 50
    kv = g.kv(3, ctx, 3 * ((ctx + 63) // 64) if paged else None, dtype=cache)
    kv.track()
    data = [(rows(2 * l, n, nkv, hd), rows(2 * l + 1, n, nkv, hd)) for l in range(3)]
    other = (rows(90, ctx, nkv, hd), rows(91, ctx, nkv, hd))
    w = [some_weights(l, nkv, n) for l in range(3)]
    for l in range(3):
        kv.write(l, 1, 0, *(on(x) for x in data[l]))
        kv.set_weights(l, 1, 0, on(w[l]))
        kv.write(l, 0, 0, *(on(x) for x in other))
        kv.write(l, 2, 0, *(on(x[:40]) for x in other))
    kv.set_len(1, n)
    kv.set_len(0, ctx)
    kv.set_len(2, 40)
    dst = 1 if in_place else 2
    kept = kv.evict(1, dst, keep, first, last, kept=True)
    evicted(kv, 3, nkv, cache, data, w, 1, dst, keep, first, last, kept)
    if paged:
        pages = lambda m: (m + 63) // 64  # noqa: E731
        assert kv.pages()[1] == 3 * pages(ctx) - pages(ctx) - pages(keep) - (pages(40) if in_place else pages(n))
    for l in range(3):
        check(kv, l, 0, 0, *(held(x, cache) for x in other), what="another user")
    kv.evict(1, dst, min(keep, kv.len(1)), 0, 0)  # without the list
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_pages_that_others_hold_stay_theirs(torch, st, cache):
    """In place on shared pages, and into a user that shares the source's; a pool that is short changes nothing."""
    g = bare_stage(st, 1, 64, layers=2)
    kv = g.kv(3, 300, 10, dtype=cache)
    kv.track()
    n = 280
    data = [(rows(2 * l, n, 1, 64), rows(2 * l + 1, n, 1, 64)) for l in range(2)]
    w = [some_weights(l, 1, n) for l in range(2)]
    for l in range(2):
        kv.write(l, 0, 0, *(on(x) for x in data[l]))
        kv.set_weights(l, 0, 0, on(w[l]))
    kv.set_len(0, n)
    kv.fork(0, 1)
    kept = kv.evict(1, 1, 150, 70, 10, kept=True)  # copies of pages 1 and 2; page 0 stays shared
    evicted(kv, 2, 1, cache, data, w, 1, 1, 150, 70, 10, kept)
    for l in range(2):
        check(kv, l, 0, 0, *(held(x, cache) for x in data[l]), what="source")
    assert kv.pages() == (10, 3)
    kv.fork(0, 2)
    kept = kv.evict(0, 2, 100, 3, 0, kept=True)
    evicted(kv, 2, 1, cache, data, w, 0, 2, 100, 3, 0, kept)
    assert kv.pages() == (10, 1)
    kv.set_len(2, 0)
    kv.fork(0, 1)
    kv.set_len(2, 300)  # every page is held
    assert kv.pages() == (10, 0)
    for call in (lambda: kv.evict(1, 1, 150, 0, 0), lambda: kv.evict(0, 1, 65, 0, 0)):
        with pytest.raises(st.KFError) as e:
            call()
        assert e.value.status == 2
        assert kv.len(1) == n and kv.pages() == (10, 0)
    for l in range(2):
        for u in (0, 1):
            check(kv, l, u, 0, *(held(x, cache) for x in data[l]))
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("first,keep", [(0, 200), (70, 201), (130, 399), (5, 400), (0, 30)])
def test_in_place_where_some_pages_are_shared(torch, st, cache, first, keep):
    """A user that shares its first pages with another and holds the rest alone; keeping everything copies nothing."""
    g = bare_stage(st, 2, 64, layers=2)
    kv = g.kv(2, 420, 14, dtype=cache)
    kv.track()
    n, own = 400, 150
    data = [(rows(2 * l, n, 2, 64), rows(2 * l + 1, n, 2, 64)) for l in range(2)]
    w = [some_weights(l, 2, n) for l in range(2)]
    for l in range(2):
        kv.write(l, 0, 0, *(on(x[:own + 50]) for x in data[l]))
    kv.set_len(0, own + 50)
    kv.fork(0, 1, own)
    for l in range(2):
        kv.write(l, 1, own, *(on(x[own:]) for x in data[l]))  # its third page is its own from here on
        kv.set_weights(l, 1, 0, on(w[l]))
    kv.set_len(1, n)
    assert kv.pages() == (14, 14 - 4 - 5)
    kept = kv.evict(1, 1, keep, first, 20, kept=True)
    evicted(kv, 2, 2, cache, data, w, 1, 1, keep, first, 20, kept)
    for l in range(2):
        check(kv, l, 0, 0, *(held(x, cache)[:own + 50] for x in data[l]), what="the other user")
    shared = 2 if keep == n else min(first // 64, 2)
    assert kv.pages() == (14, 14 - 4 - ((keep + 63) // 64 - min(shared, (keep + 63) // 64)))
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("n,keep", [(4000, 1999), (4097, 4000), (20000, 5001), (40000, 30000)])
def test_lists_of_every_length(torch, st, n, keep):
    """The positions kept of rows that a workgroup holds in registers, in each size of them, and of a longer one; in place,
    where moves wait for each other."""
    g = bare_stage(st, 3, 64)
    kv = g.kv(2, n)
    kv.track()
    w = some_weights(5, 3, n)
    x = np.arange(n, dtype=np.float32)[:, None, None] % 2048 * np.ones((1, 3, 64), np.float32)
    y = np.arange(n, dtype=np.float32)[:, None, None] // 2048 * np.ones((1, 3, 64), np.float32)
    kv.write(0, 0, 0, on(x), on(y))
    kv.set_weights(0, 0, 0, on(w))
    kv.set_len(0, n)
    apart = kv.evict(0, 1, keep, 100, 300, kept=True)
    kept = kv.evict(0, 0, keep, 100, 300, kept=True)
    assert torch.equal(apart, kept)
    for u in (1, 0):
        a, b = kv.read(0, u, 0, keep)
        at = (b * 2048 + a)[:, :, 0].t().int()
        assert torch.equal(at, kept[0])
        assert all(torch.equal(t[:, :, :1].expand_as(t), t) for t in (a, b))
    for g_ in range(3):
        assert kept[0, g_].tolist() == kept_of(w[g_].tolist(), keep, 100, 300)
    kv.close()
    g.close()


@pytest.mark.parametrize("n,equal", [(30000, 30000), (30000, 20000), (8192, 8192), (200, 200)])
def test_many_equal_weights(torch, st, n, equal):
    """More equal weights than a list of them holds, in rows that a workgroup has in registers: the lower positions stay."""
    g = bare_stage(st, 1, 64)
    kv = g.kv(1, n)
    kv.track()
    w = np.full((1, n), 0.5, np.float32)
    w[0, np.random.default_rng(n).permutation(n)[equal:]] = np.float32(0.5) + np.arange(n - equal, dtype=np.float32) % 7 * np.float32(2.0 ** -20)
    kv.set_weights(0, 0, 0, on(w))
    for keep, first, last in ((n // 3, 0, 0), (n - 1, 1, 2), (n // 2, 20, n // 4), (n, 3, 4)):
        kv.set_len(0, n)
        kv.write(0, 0, 0, *[torch.zeros((n, 1, 64), device="cuda")] * 2)
        kv.set_weights(0, 0, 0, on(w))
        kept = kv.evict(0, 0, keep, first, last, kept=True)
        assert kept[0, 0].tolist() == kept_of(w[0].tolist(), keep, first, last), (keep, first, last)
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_weights_of_replaced_pages(torch, st, cache):
    """In place where all pages are shared: none of them is written, but the weights of the positions they hold are moved
    within their row, behind those that still read there."""
    n, keep, nkv, layers = 6000, 2500, 8, 4
    g = bare_stage(st, nkv, 64, layers=layers)
    pages = (n + 63) // 64
    kv = g.kv(2, n, pages + (keep + 63) // 64, dtype=cache)
    kv.track()
    x = torch.ones((n, nkv, 64), device="cuda")
    w = [np.random.default_rng(l).permutation(nkv * n).reshape(nkv, n).astype(np.float32) for l in range(layers)]
    for l in range(layers):
        kv.write(l, 0, 0, x, x)
        kv.set_weights(l, 0, 0, on(w[l]))
    kv.set_len(0, n)
    for _ in range(5):
        kv.fork(0, 1)
        kept = kv.evict(1, 1, keep, 10, 100, kept=True).cpu().numpy()
        for l in range(layers):
            assert np.array_equal(kv.weights(l, 1, 0, keep).cpu().numpy(), np.take_along_axis(w[l], kept[l].astype(np.int64), 1)), l
    for g_ in range(nkv):
        assert kept[0, g_].tolist() == kept_of(w[0][g_].tolist(), keep, 10, 100)
    kv.close()
    g.close()


def test_a_long_eviction(torch, st):
    """262144 positions of one head, nearly all weights equal or different, half of them kept."""
    n, keep = 262144, 131001
    g = bare_stage(st, 2, 64)
    kv = g.kv(2, n)
    kv.track()
    r = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((n, 2, 64), device="cuda").normal_(generator=r).half()
    kv.write(0, 0, 0, x, x)
    kv.set_len(0, n)
    w = torch.rand((2, n), device="cuda", generator=r)
    w[1] = torch.where(w[1] < 0.9, 0.25, w[1])
    kv.set_weights(0, 0, 0, w)
    kept = kv.evict(0, 1, keep, 4, 1000, kept=True)[0].long()
    for g_ in range(2):
        assert kept[g_].tolist() == kept_of(w[g_].tolist(), keep, 4, 1000)
        assert torch.equal(kv.read(0, 1, 0, keep)[0][:, g_], x[kept[g_], g_].float())
    again = kv.evict(0, 0, keep, 4, 1000, kept=True)[0]
    assert torch.equal(again.long(), kept)
    assert all(torch.equal(a, b) for a, b in zip(kv.read(0, 0, 0, keep), kv.read(0, 1, 0, keep)))
    assert torch.equal(kv.weights(0, 0, 0, keep), kv.weights(0, 1, 0, keep))
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_drafts_and_evictions_together(torch, st, cache):
    """A user as a server of long contexts keeps it: a prompt weighed by its last queries and evicted to its budget, then
    drafts that are written, attended to and accepted in part, weighed, and evicted again, beside a second user that
    shares the prompt; every attention and all that the cache holds against 64 bits."""
    hd, nkv, group, n, budget = 64, 2, 4, 500, 300
    g = bare_stage(st, nkv, hd, layers=2, group=group)
    kv = g.kv(2, 700, 22, dtype=cache)
    kv.track()
    model = [[held(rows(2 * l + i, n, nkv, hd), cache) for i in range(2)] for l in range(2)]  # [layer] k, v
    for l in range(2):
        kv.write(l, 0, 0, *(on(rows(2 * l + i, n, nkv, hd)) for i in range(2)))
    kv.set_len(0, n)
    kv.fork(0, 1)
    prompt = [[x.copy() for x in m] for m in model]
    weights = [np.zeros((nkv, n)) for _ in range(2)]

    def weigh(l, lens, seed):
        q = rows(seed, len(lens), nkv * group, hd)
        kv.weigh(l, [0] * len(lens), lens, on(q))
        for b, m in enumerate(lens):
            weights[l] += weight_of(q[b], model[l][0], m)[0]

    def evict(keep):
        kept = kv.evict(0, 0, keep, 4, 32, kept=True).cpu().numpy()
        for l in range(2):
            for h in range(nkv):
                # as the library's own sums have it, which are near the model's
                lo = weights[l][h][np.setdiff1d(np.arange(weights[l].shape[1]), kept[l, h])]
                assert lo.max(initial=0) <= weights[l][h][kept[l, h][4:-32]].min() * (1 + 1e-4)
                assert np.array_equal(kept[l, h][:4], np.arange(4)) and np.all(np.diff(kept[l, h]) > 0)
            pick = lambda x: np.stack([x[kept[l, h], h] for h in range(nkv)], 1)  # noqa: E731
            model[l] = [pick(x) for x in model[l]]
            weights[l] = np.stack([weights[l][h][kept[l, h]] for h in range(nkv)])

    for l in range(2):
        weigh(l, [n - 7 + i for i in range(8)], 50 + l)
    evict(budget)
    for step in range(6):
        length, m = kv.len(0), 20 + 13 * step
        par = draft(step, m)
        path, j = [], m - 1  # the last token's ancestors
        while j >= 0:
            path.insert(0, j)
            j = par[j]
        p = torch.tensor(par, dtype=torch.int32, device="cuda")
        for l in range(2):
            new = [rows(1000 + 10 * step + 2 * l + i, m, nkv, hd) for i in range(2)]
            kv.write(l, 0, length, *(on(x) for x in new))
            q = rows(2000 + 10 * step + l, m, nkv * group, hd)
            got = kv.attend_tree(l, [0], [length], [m], p, on(q)).double().cpu().numpy()
            k, v = (np.concatenate([a, held(b, cache)]) for a, b in zip(model[l], new))
            # tests/test_gpu_tree.py's bound at values and scores of this size
            assert np.abs(got - want_of(q, k, v, length, par)).max() < 1e-4
            model[l] = [np.concatenate([a, held(b, cache)[path]]) for a, b in zip(model[l], new)]
            weights[l] = np.concatenate([weights[l], np.zeros((nkv, len(path)))], 1)
        kv.accept(0, length, path)
        assert kv.len(0) == length + len(path)
        for l in range(2):
            weigh(l, [kv.len(0)], 3000 + 10 * step + l)
            got = kv.weights(l, 0, 0, kv.len(0)).double().cpu().numpy()
            assert np.abs(got - weights[l]).max() < 1e-4
            check(kv, l, 0, 0, *model[l], what=f"step {step}")
        if step % 2:
            evict(budget)
    for l in range(2):
        check(kv, l, 1, 0, *prompt[l], what="second user")
    g.sync()
    kv.close()
    g.close()


def test_refusals(torch, st):
    g = bare_stage(st, 1, 64, layers=2, group=2)
    kv, paged = g.kv(2, 100), g.kv(2, 100, 3)
    q, w = on(rows(3, 2, 2, 64)), torch.zeros((1, 10), device="cuda")

    def refused(status, call, *args):
        with pytest.raises(st.KFError) as e:
            call(*args)
        assert e.value.status == status
    # untracked
    refused(4, kv.weigh, 0, [0], [1], q[:1])
    refused(4, kv.weights, 0, 0, 0, 10)
    refused(4, kv.set_weights, 0, 0, 0, w)
    refused(4, kv.evict, 0, 0, 0)
    refused(1, kv.track, -1)
    refused(1, kv.track, 33)
    for c in (kv, paged):
        c.track(32)
        c.track()
    paged.write(0, 0, 0, on(rows(1, 64, 1, 64)), on(rows(2, 64, 1, 64)))
    refused(3, paged.weigh, 0, [0, 0], [64, 65], q)
    refused(3, paged.weigh, 0, [0, 1], [64, 1], q)
    refused(3, kv.weigh, 0, [0, 0], [64, 101], q)
    refused(1, kv.weigh, 0, [0, 0], [64, -1], q)
    refused(1, kv.weigh, 0, [0, 2], [64, 1], q)
    refused(1, kv.weigh, 2, [0, 1], [64, 1], q)
    refused(1, kv.weigh, 0, [], [], q[:0])
    refused(1, kv.weigh, 0, [0] * 33, [1] * 33, torch.zeros((33, 2, 64), device="cuda"))
    refused(1, kv.weigh, 0, [0], [1], torch.zeros(129, device="cuda")[1:].view(1, 2, 64))
    refused(3, kv.weights, 0, 0, 91, 10)
    refused(1, kv.weights, 0, 2, 0, 10)
    refused(1, kv.weights, 2, 0, 0, 10)
    refused(3, kv.set_weights, 0, 0, 91, w)
    refused(1, kv.set_weights, 0, 0, -1, w)
    kv.set_len(0, 50)
    refused(3, kv.evict, 0, 1, 51)
    refused(1, kv.evict, 0, 2, 5)
    refused(1, kv.evict, -1, 0, 5)
    refused(1, kv.evict, 0, 1, -1)
    refused(1, kv.evict, 0, 1, 10, 6, 5)
    refused(1, kv.evict, 0, 1, 10, -1, 5)
    refused(1, kv.evict, 0, 1, 10, 1, -5)
    for bad in (w.double(), w[0], torch.zeros((2, 10), device="cuda")):
        with pytest.raises(ValueError):
            kv.set_weights(0, 0, 0, bad)
    with pytest.raises(ValueError):
        kv.weigh(0, [0], [1, 2], q[:1])
    with pytest.raises(TypeError):
        kv.weigh(0, [0, 0], [1, 2], q.double())
    assert kv.len(0) == 50 and kv.len(1) == 0 and paged.pages() == (3, 2)
    assert not kv.weights(0, 0, 0, 100).any()
    g.sync()
    kv.close()
    paged.close()
    g.close()


def test_captured_weighing_and_eviction(torch, st):
    """A captured weighing and eviction reads queries and cache as they are at each replay, on another stream, among eager
    calls on the same workspace; on a paged cache an eviction under capture is refused."""
    hd, nkv, group, n = 128, 2, 4, 2000
    g = bare_stage(st, nkv, hd, group=group)
    kv, paged = g.kv(2, n), g.kv(1, 100, 2)
    kv.track()
    paged.track()
    paged.set_len(0, 100)
    kv.set_len(0, n)
    kvs = [[on(rows(10 * i + j, n, nkv, hd)) for j in range(2)] for i in range(3)]
    qs = [on(rows(90 + i, 5, nkv * group, hd)) for i in range(3)]
    k, v, q = (t.clone() for t in (*kvs[0], qs[0]))
    kept = torch.empty((1, nkv, 300), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)

    def step(k, v, q):
        kv.write(0, 0, 0, k, v)
        kv.weigh(0, [0] * 5, [n, 10, n, 0, 1999], q)
        st._check(kv._lib.kf_kv_evict(kv.handle, 0, 1, 300, 5, 20, kept.data_ptr()), "kf_kv_evict")
    with torch.cuda.stream(side):
        eager = []
        for i in range(3):
            step(*kvs[i], qs[i])
            eager.append((kept.clone(), kv.weights(0, 0, 0, n).clone(), *(t.clone() for t in kv.read(0, 1, 0, 300))))
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(k, v, q)
            with pytest.raises(st.KFError) as e:
                paged.evict(0, 0, 10)
            assert e.value.status == 4
        for i in (1, 0, 2, 1):
            for t, x in zip((k, v, q), (*kvs[i], qs[i])):
                t.copy_(x)
            graph.replay()
            got = (kept, kv.weights(0, 0, 0, n), *kv.read(0, 1, 0, 300))
            kv.attend(0, [0], [n], qs[i][:1].contiguous())
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, eager[i])), i
    assert paged.len(0) == 100
    g.sync()
    kv.close()
    paged.close()
    g.close()


def test_captured_decode_steps_on_a_tracked_cache(torch, st):
    """Replayed steps give the weights of eager ones."""
    shape = synth.SHAPE_TINY
    model = SeededModel(shape, 73)
    g = st.Stage(shape, 0, 2, model.layer)
    g.set_flags(st.KF_STAGE_ORDERED)
    kv = g.kv(1, 300)
    kv.track(4)
    h = on(synth.hidden_states(73, synth.STREAM_PREFILL_HIDDEN, 0, 100, shape.hidden))
    xs = [on(synth.hidden_states(73, synth.STREAM_DECODE_HIDDEN, i, 1, shape.hidden)) for i in range(3)]
    x, y = xs[0].clone(), torch.empty_like(xs[0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)
    with torch.cuda.stream(side):
        def prompt():
            kv.set_len(0, 0)
            g.prefill(kv, 0, 0, hidden=h)
        eager = []
        for t in xs:
            prompt()
            g.decode(kv, [0], [100], hidden=t)
            eager.append([kv.weights(l, 0, 0, 101).clone() for l in range(2)])
        prompt()
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            g.decode(kv, [0], [100], hidden=x, out=y)
        for i in (2, 0, 1):
            prompt()
            x.copy_(xs[i])
            graph.replay()
            got = [kv.weights(l, 0, 0, 101) for l in range(2)]
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, eager[i])), i
    g.sync()
    kv.close()
    g.close()


def layer64(x, w, shape, k, v, new, rot):
    """One layer in 64 bits over rows x at rotations rot; row i sees the cached keys and values [.., nkv, hd] up to `new` + i,
    which hold the rows' own.  Returns the rows' outputs, queries and keys."""
    hd = shape.head_dim
    xn = so.rms_norm(x, w["attn_norm"], shape.rms_eps)
    q, key = ((xn @ w[n].T).reshape(len(x), -1, hd) for n in ("wq", "wk"))
    if shape.qk_norm:
        q, key = so.rms_norm(q, w["q_norm"], shape.rms_eps), so.rms_norm(key, w["k_norm"], shape.rms_eps)
    q, key = so.rope(q, np.asarray(rot), shape.rope_theta), so.rope(key, np.asarray(rot), shape.rope_theta)
    upto = [new + i + 1 for i in range(len(x))]
    x = x + so.attention_rows(q, [k[:n] for n in upto], [v[:n] for n in upto], shape.n_kv_heads) @ w["wo"].T
    return x + so.mlp_swiglu(so.rms_norm(x, w["mlp_norm"], shape.rms_eps), w["wg"], w["wu"], w["wd"]), q, key


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("shape", [synth.ModelShape(2, 512, 8, 2, 64, 1408, 1000), synth.ModelShape(2, 384, 8, 2, 64, 1024, 1000, qk_norm=True),
                                   synth.ModelShape(2, 512, 8, 2, 128, 704, 0, qk_norm=True)], ids=["tiny", "qwen3", "hd128"])
def test_tokens_after_an_eviction_keep_their_distances(torch, st, cache, shape):
    """A prompt is cut, then decode steps (alone and beside a user that lost nothing), a chunk, a second cut that takes the
    rotations past max_ctx, and a step of a fork: every token is rotated as if nothing had been dropped."""
    cfg, n, ctx = 77, 150, 160
    model = SeededModel(shape, cfg)
    w = [{k: so.bf16_to_f64(v) for k, v in model.layer(l).items()} for l in range(2)]
    g = st.Stage(shape, 0, 2, model.layer)
    kv = g.kv(3, ctx, 12, dtype=cache)
    kv.track(8)
    for u in range(2):
        g.prefill(kv, u, 0, hidden=on(synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, u, n - 80 * u, shape.hidden)))
    assert [kv.dropped(u) for u in range(3)] == [0, 0, 0]
    seen = [n, n - 80, 0]  # tokens of each user's text

    def compare(user, x, got, m):
        """The last m tokens of the user, whose outputs are `got`; what they attend to is read back."""
        new = kv.len(user) - m
        assert seen[user] - kv.dropped(user) == new
        rot = [seen[user] + i for i in range(m)]
        x = np.asarray(x, np.float64)
        for l in range(2):
            k, v = (t.double().cpu().numpy() for t in kv.read(l, user, 0, new + m))
            x, q, key = layer64(x, w[l], shape, k, v, new, rot)
            # fp16 operands and cache: some 2^-10 of the largest.  A 4-bit block's largest value is M < 7 units, its codes end
            # in 3, 4 and 6: a value up to 4 is off by 1/2 at most and M is 3.5 at least, so by M / 7; one of 4 to 5 by what
            # it has beyond 4, (M - 4) / M <= 1/5 of M at M = 5; one past 5 by 1, 1/5 of M at most.
            assert np.abs(k[new:] - key).max() <= (3e-3 if cache == "f16" else 0.2 + 3e-3) * np.abs(key).max(), (user, l)
            if m == 1:
                # a query off by 2^-8 (a layer's fp16 operands) moves a score by that of its sum of |products|
                a, _ = weight_of(q[0], k, new + 1)
                G = shape.n_q_heads // shape.n_kv_heads
                S = max((np.abs(k[:, h // G]) @ np.abs(q[0, h])).max() for h in range(shape.n_q_heads)) / math.sqrt(shape.head_dim)
                b = kv.weights(l, user, 0, new + 1).double().cpu().numpy() - before[user, l]
                assert np.all(np.abs(a - b) <= a * math.expm1(2 * 2.0 ** -8 * S) + 1e-5), (user, l)
        got = got.double().cpu().numpy()
        assert np.all(np.abs(got - x).max(1) <= 1e-2 * np.abs(x).max(1)), user
        seen[user] += m

    def decode(step, users):
        x = synth.hidden_states(cfg, synth.STREAM_DECODE_HIDDEN, step, len(users), shape.hidden)
        for u in users:
            for l in range(2):
                old = kv.weights(l, u, 0, kv.len(u)).double().cpu().numpy()
                before[u, l] = np.concatenate([old, np.zeros((shape.n_kv_heads, 1))], 1)
        out = g.decode(kv, users, [kv.len(u) for u in users], hidden=on(x))
        for i, u in enumerate(users):
            compare(u, x[i:i + 1], out[i:i + 1], 1)
    before = {}
    kv.evict(0, 0, 90, 4, 20)
    assert kv.dropped(0) == 60 and kv.len(0) == 90
    decode(0, [0])
    decode(1, [0, 1])
    x = synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, 7, 33, shape.hidden)
    compare(0, x, g.prefill(kv, 0, kv.len(0), hidden=on(x), noalloc=True), 33)
    kv.evict(0, 0, 50, 4, 20)  # the next token's rotation is past max_ctx
    assert kv.dropped(0) == 60 + 125 - 50 and seen[0] > ctx
    decode(2, [1, 0])
    kv.fork(0, 2)
    seen[2] = seen[0]
    assert kv.dropped(2) == kv.dropped(0)
    decode(3, [2])
    kv.evict(0, 2, 10, 1, 9)
    seen[2] = seen[0]
    decode(4, [2, 0])
    kv.set_len(2, 0)
    assert kv.dropped(2) == 0
    other = g.kv(1, ctx, dtype=cache)
    other.copy(kv, 0, 0, 5, 10)
    assert other.dropped(0) == 0
    other.copy(kv, 0, 0, 0, 20)
    assert other.dropped(0) == kv.dropped(0)
    other.set_dropped(0, 7)
    assert other.dropped(0) == 7
    for bad in (-1, 2 ** 31 - ctx):
        with pytest.raises(st.KFError) as e:
            other.set_dropped(0, bad)
        assert e.value.status == st.KF_ERANGE
    with pytest.raises(st.KFError):
        other.dropped(1)
    g.sync()
    kv.close()
    other.close()
    g.close()


def test_rotations_that_a_capture_cannot_allocate(torch, st):
    """A captured eviction leaves the table of rotations as it is: a captured step or a chunk without allocations that needs
    more is refused with nothing changed, and an eager step makes it."""
    shape = synth.ModelShape(1, 512, 8, 2, 64, 1408, 1000)
    model = SeededModel(shape, 5)
    g = st.Stage(shape, 0, 1, model.layer)
    n = 100
    kv = g.kv(2, n)
    kv.track()
    g.prefill(kv, 0, 0, hidden=on(synth.hidden_states(5, synth.STREAM_PREFILL_HIDDEN, 0, n, shape.hidden)))
    x = on(synth.hidden_states(5, synth.STREAM_DECODE_HIDDEN, 0, 1, shape.hidden))
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kv.evict(0, 1, 40, 2, 30)
            with pytest.raises(st.KFError) as e:
                g.decode(kv, [1], [40], hidden=x, out=out)
            assert e.value.status == st.KF_ESTATE
        for _ in range(3):
            graph.replay()
            side.synchronize()
        assert (kv.len(1), kv.dropped(1)) == (40, 60)
        with pytest.raises(st.KFError) as e:
            g.prefill(kv, 1, 40, hidden=x, out=out, noalloc=True)
        assert e.value.status == st.KF_ESTATE and kv.len(1) == 40
        w = {k: so.bf16_to_f64(v) for k, v in model.layer(0).items()}
        for step in range(2):
            g.decode(kv, [1], [40 + step], hidden=x, out=out)
            k, v = (t.double().cpu().numpy() for t in kv.read(0, 1, 0, 41 + step))
            want, _, key = layer64(x.double().cpu().numpy(), w, shape, k, v, 40 + step, [n + step])
            assert np.abs(k[40 + step:] - key).max() <= 3e-3 * np.abs(key).max()
            assert np.abs(out.double().cpu().numpy() - want).max() <= 1e-2 * np.abs(want).max()
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("shape", [synth.ModelShape(1, 512, 8, 2, 64, 704, 0), synth.ModelShape(1, 512, 8, 2, 128, 704, 0, qk_norm=True)],
                         ids=["hd64", "hd128"])
def test_tracked_steps_over_many_splits(torch, st, cache, shape):
    """A step's weights come from its attention's own maxima and sums, of one split or of many, in batches of very different
    lengths."""
    model = SeededModel(shape, 11)
    w = {k: so.bf16_to_f64(v) for k, v in model.layer(0).items()}
    g = st.Stage(shape, 0, 1, model.layer)
    lens = [20000, 70, 0, 4097]
    kv = g.kv(4, max(lens) + 8, dtype=cache)
    kv.track()
    for u, n in enumerate(lens):
        if n:
            kv.write(0, u, 0, on(rows(u, n, 2, shape.head_dim)), on(rows(9 + u, n, 2, shape.head_dim)))
        kv.set_len(u, n)
    for step, users in enumerate(([0], [3, 0], [2, 0, 1, 3], [1])):
        x = synth.hidden_states(11, synth.STREAM_DECODE_HIDDEN, step, len(users), shape.hidden)
        before = [kv.weights(0, u, 0, kv.len(u) + 1).double().cpu().numpy() for u in users]
        at = [kv.len(u) for u in users]
        g.decode(kv, users, at, hidden=on(x))
        for i, u in enumerate(users):
            n = at[i] + 1
            k, v = (t.double().cpu().numpy() for t in kv.read(0, u, 0, n))
            _, q, _ = layer64(np.asarray(x[i:i + 1], np.float64), w, shape, k, v, at[i], [at[i]])
            before[i][:, at[i]] = 0
            a, e = weight_of(q[0], k, n)
            # as test_prefill_and_decode_steps_add_theirs has it, and the fp16 probabilities whose sum the attention takes
            # (2^-11 of each, and 2^-25 of the largest where they end)
            G = shape.n_q_heads // shape.n_kv_heads
            S = max((np.abs(k[:, h // G]) @ np.abs(q[0, h])).max() for h in range(shape.n_q_heads)) / math.sqrt(shape.head_dim)
            tol = e + a * (math.expm1(2 * 2 * 2.0 ** -11 * S) + 2.0 ** -11 + n * 2.0 ** -25) + 2.0 ** -24 * (1 + before[i])
            got = kv.weights(0, u, 0, n).double().cpu().numpy() - before[i]
            assert np.all(np.abs(got - a) <= tol), (step, u)
    g.sync()
    kv.close()
    g.close()
