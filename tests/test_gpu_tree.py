"""Attention of trees of drafted tokens over a cache (kf_kv_attend_tree) and accepted paths (kf_kv_accept)."""
import math
import random

import numpy as np
import pytest

from tests.test_gpu_attend import EPS, on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_cache import bare_stage, check, held, rows

pytestmark = pytest.mark.gpu


def sees(parents):
    """[n, n]: which tokens each token attends to, by walking up from each."""
    n = len(parents)
    m = np.zeros((n, n), bool)
    for i in range(n):
        j = i if parents[i] != -2 else -1
        while j >= 0:
            if parents[j] != -2:
                m[i, j] = True
            j = parents[j] if 0 <= parents[j] < j else -1
    return m


def want_of(q, k, v, length, parents):
    """The attention of a tree's tokens q [n, nq, hd] over k, v [length + n, nkv, hd] in 64 bits."""
    n, nq, hd = q.shape
    nkv = k.shape[1]
    m = np.concatenate([np.repeat(np.array(parents)[:, None] != -2, length, 1), sees(parents)], 1)
    out = np.zeros((n, nq, hd))
    for i in range(n):
        at = np.flatnonzero(m[i])
        for h in range(nq if len(at) else 0):
            g = h // (nq // nkv)
            s = k[at, g] @ q[i, h].astype(np.float64) / math.sqrt(hd)
            p = np.exp(s - s.max())
            out[i, h] = p @ v[at, g] / p.sum()
    return out


def allowed(q, k, v, want, io):
    """How far outputs may be off, [n, nq, 1].

    With scores in log2 units and S the largest sum of |products| of a score: a score is off by the query's rounding (two
    fp16 parts, 2^-22; none for 16-bit queries) and by hd + 4 fp32 roundings (2^-24 S each).  A probability is off by ln 2 of
    that, 2^-22 for the exponential and its own rounding: 2^-22 in two fp16 parts, 2^-11 in one (bfloat16).  Numerator and
    denominator each by that and 2^-24 for each addition along a chain (fewer than 200, the sums being split), relative to
    sum p |v|; the output's own rounding comes on top."""
    n, nq, hd = q.shape
    nkv = k.shape[1]
    kk = np.abs(k).max(0).repeat(nq // nkv, 0)  # [nq, hd]
    S = (np.abs(q.astype(np.float64)) * kk).sum(-1) * math.log2(math.e) / math.sqrt(hd)
    rel = math.log(2) * S * (2.0 ** -22 + (hd + 4) * 2.0 ** -24) + 2.0 ** -22 + 200 * 2.0 ** -24
    rel = rel + (2.0 ** -11 if io == "bfloat16" else 2.0 ** -22)
    most = np.abs(v).max((0, 2)).repeat(nq // nkv)
    return (2 * rel * most + EPS[io] * np.abs(want).max(-1))[..., None] * 1.01


def draft(seed, n):
    r = random.Random(seed)
    return [max(i - 1 - int(r.expovariate(0.3)), -1) for i in range(n)]


CHAIN = list(range(-1, 255))
SHAPES = [
    # hd, nkv, group, [(cached positions, parents)], paged
    (128, 2, 4, [(200, draft(1, 26))], False),
    (64, 2, 4, [(0, [-1]), (1, draft(2, 7)), (63, draft(3, 70)), (64, [-1, 0, 0, -2, 2, 3])], True),
    (128, 1, 8, [(3000, draft(4, 64)), (127, draft(5, 256))], True),
    (64, 3, 1, [(0, draft(6, 130))], False),
    (128, 2, 5, [(1000, CHAIN), (129, [-1] * 65)], False),
    (64, 1, 8, [(1500, [])], True),
    (64, 1, 7, [(65, [-2, -2]), (31, draft(7, 33)), (5, [5, 0, 7, 2, -9, 1 << 30, 3])], True),  # parents that are no earlier token
    (128, 8, 1, [(2, draft(8, 3)), (700, draft(9, 15)), (1100, [-1]), (1023, draft(10, 129))], False)]


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("io", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_against_64_bits(torch, st, cache, io, case):
    """Trees of every form behind lengths around pages, rows that pad, with other values in the cache behind each tree."""
    hd, nkv, group, trees, paged = SHAPES[case]
    users, lens, nodes = [3 - b for b in range(len(trees))], [t[0] for t in trees], [len(t[1]) for t in trees]
    ctx = max(a + n for a, n in zip(lens, nodes)) + 100
    g = bare_stage(st, nkv, hd, layers=2, group=group)
    kv = g.kv(4, ctx, 4 * ((ctx + 63) // 64) if paged else None, dtype=cache)
    q = on(rows(5, sum(nodes), nkv * group, hd, 1.5), getattr(torch, io))
    parents = torch.tensor([p for t in trees for p in t[1]], dtype=torch.int32, device="cuda")
    want, tol, at = [], [], 0
    for b, (n, par) in enumerate(trees):
        k, v = rows(10 + b, ctx, nkv, hd, 2.0), rows(20 + b, ctx, nkv, hd)
        kv.write(1, users[b], 0, on(k), on(v))
        k, v = held(k, cache)[:n + len(par)], held(v, cache)[:n + len(par)]
        qb = q[at:at + len(par)].float().cpu().numpy()
        at += len(par)
        want.append(want_of(qb, k, v, n, par))
        tol.append(allowed(qb, k, v, want[-1], io))
    got = kv.attend_tree(1, users, lens, nodes, parents, q)
    assert got.dtype == q.dtype and got.shape == q.shape
    want, tol = np.concatenate(want), np.concatenate(tol)
    err = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
    assert np.all(err <= tol), (err / np.maximum(tol, 1e-300)).max()
    assert not got[parents == -2].any()
    assert torch.equal(kv.attend_tree(1, users, lens, nodes, parents, q), got)
    kv.attend_tree(1, users, lens, nodes, parents, q, out=q)  # in place
    assert torch.equal(q, got)
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("io", ["float32", "bfloat16"])
def test_a_single_token_is_attention_with_one_more_position(torch, st, cache, io):
    """A tree of one token gives what kf_kv_attend gives over len + 1 positions, and several rows of one user may repeat it."""
    hd, nkv, group, n = 128, 2, 4, 500
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(1, n + 1, dtype=cache)
    k, v = rows(1, n + 1, nkv, hd), rows(2, n + 1, nkv, hd)
    kv.write(0, 0, 0, on(k), on(v))
    q = on(rows(3, 2, nkv * group, hd), getattr(torch, io))
    root = torch.full((2,), -1, dtype=torch.int32, device="cuda")
    got = kv.attend_tree(0, [0, 0], [n, 37], [1, 1], root, q)
    want = kv.attend(0, [0, 0], [n + 1, 38], q)
    for b, m in enumerate((n + 1, 38)):
        qb = q[b:b + 1].float().cpu().numpy()
        tol = 2 * allowed(qb, held(k, cache)[:m], held(v, cache)[:m], want[b:b + 1].double().cpu().numpy(), io)
        assert np.all(np.abs((got[b] - want[b]).double().cpu().numpy()) <= tol[0])
    kv.close()
    g.close()


@pytest.mark.parametrize("io", ["float32", "bfloat16"])
def test_what_a_token_does_not_see_does_not_reach_it(torch, st, io):
    """Infinities and NaN among the keys and values of tokens that others do not see, and behind the tree: the others
    are as without them, and the tokens that see them get what the formula gives."""
    hd, nkv, group, n, m = 128, 2, 4, 150, 20
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(1, n + m + 30)
    k, v = rows(1, n + m + 30, nkv, hd), rows(2, n + m + 30, nkv, hd)
    parents = [-1] + [0] * 9 + [1, 2, 3, 4, 5, -2, 10, 11, 12, 13]
    p = torch.tensor(parents, dtype=torch.int32, device="cuda")
    q = on(rows(3, m, nkv * group, hd), getattr(torch, io))
    kv.write(0, 0, 0, on(k), on(v))
    clean = kv.attend_tree(0, [0], [n], [m], p, q)
    v[n + 6, 0, 5], v[n + 6, 0, 6], v[n + 6, 1, 7] = np.inf, -np.inf, np.nan  # a leaf of the root
    v[n + 7, 0, 5], v[n + 7, 1, 100] = -np.inf, 1e30
    k[n + 8, 1, 3] = np.nan
    k[n + 15], v[n + 15] = np.inf, np.nan                                   # the row that pads
    k[n + m:], v[n + m:] = np.nan, np.inf                                   # behind the tree
    kv.write(0, 0, 0, on(k), on(v))
    got = kv.attend_tree(0, [0], [n], [m], p, q)
    others = [i for i in range(m) if i not in (6, 7, 8)]
    assert torch.equal(got[others], clean[others])
    want = clean.clone()
    want[6, :group, 5], want[6, :group, 6], want[6, group:, 7] = math.inf, -math.inf, math.nan
    want[7, :group, 5], want[7, group:, 100] = -math.inf, math.inf
    want[8, group:] = math.nan
    assert torch.equal(torch.nan_to_num(got, nan=7.0), torch.nan_to_num(want, nan=7.0))
    # two infinities of either sign in one place that a token sees
    v[n + 1, 0, 9], v[n + 10, 0, 9] = np.inf, -np.inf
    kv.write(0, 0, 0, on(k), on(v))
    got = kv.attend_tree(0, [0], [n], [m], p, q)
    assert torch.isposinf(got[1, :group, 9]).all() and torch.isnan(got[10, :group, 9]).all() and torch.isnan(got[16, :group, 9]).all()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_a_query_that_is_not_finite_stays_in_its_head(torch, st, cache):
    g = bare_stage(st, 1, 64, group=4)
    kv = g.kv(1, 700, dtype=cache)
    kv.write(0, 0, 0, on(rows(1, 700, 1, 64)), on(rows(2, 700, 1, 64)))
    q, p = on(rows(3, 40, 4, 64)), torch.tensor(draft(1, 40), dtype=torch.int32, device="cuda")
    clean = kv.attend_tree(0, [0], [600], [40], p, q)
    q[0, 2, 7], q[33, 0, 1] = math.nan, math.inf
    got = kv.attend_tree(0, [0], [600], [40], p, q)
    bad = torch.zeros(40, 4, dtype=torch.bool, device="cuda")
    bad[0, 2] = bad[33, 0] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])
    kv.close()
    g.close()


@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_queries_of_any_size(torch, st, size):
    """fp32 queries far from 1: the smallest give the mean of what a token sees, the largest its best key's value."""
    n, m = 300, 9
    g = bare_stage(st, 1, 64, group=2)
    kv = g.kv(1, n + m)
    k, v = rows(1, n + m, 1, 64), rows(2, n + m, 1, 64)
    kv.write(0, 0, 0, on(k), on(v))
    par = draft(3, m)
    q = rows(4, m, 2, 64) * np.float32(size)
    got = kv.attend_tree(0, [0], [n], [m], torch.tensor(par, dtype=torch.int32, device="cuda"), on(q)).double().cpu().numpy()
    k, v = held(k, "f16"), held(v, "f16")
    want = want_of(q, k, v, n, par)
    assert np.all(np.abs(got - want) <= allowed(q * (size < 1), k, v, want, "float32"))
    kv.close()
    g.close()


def test_a_long_context(torch, st):
    """Splits of several blocks, past 64 pages each, at positions whose offsets pass 32 bits."""
    hd, nkv, group, n, m = 128, 8, 2, (1 << 20) - 200, 200
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(2, 1 << 20)
    at = [(0, 3), (70_001, 64), (n - 40, 40 + m)]
    parts = [(rows(2 * i, c, nkv, hd), rows(2 * i + 1, c, nkv, hd, 1e3)) for i, (_, c) in enumerate(at)]
    for (pos, _), (k, v) in zip(at, parts):
        kv.write(0, 1, pos, on(k), on(v))
    par = draft(2, m)
    q = rows(9, m, nkv * group, hd, 2.0)
    got = kv.attend_tree(0, [1], [n], [m], torch.tensor(par, dtype=torch.int32, device="cuda"), on(q)).double().cpu().numpy()
    # the other positions' keys and values are zero: score 0 each, and nothing added
    k, v = (np.concatenate([held(x[i], "f16") for x in parts]) for i in (0, 1))
    m0 = len(k) - m
    zeros = n - m0
    mask = np.concatenate([np.ones((m, m0), bool), sees(par)], 1)
    want, tol = np.zeros_like(got), np.zeros(got.shape[:2] + (1,))
    for i in range(m):
        for h in range(nkv * group):
            s = k[mask[i], h // group] @ q[i, h].astype(np.float64) / math.sqrt(hd)
            top = max(s.max(), 0.0)
            p = np.exp(s - top)
            total = p.sum() + zeros * np.exp(-top)
            want[i, h] = p @ v[mask[i], h // group] / total
            # as `allowed`, of the part that these positions have; chains of 1300 additions: 64 positions of up to 37 blocks a
            # split in the products (four to an addition), and the merge
            S = np.abs(k[mask[i], h // group]) @ np.abs(q[i, h].astype(np.float64)) * math.log2(math.e) / math.sqrt(hd)
            rel = math.log(2) * S.max() * (2.0 ** -22 + (hd + 4) * 2.0 ** -24) + 2 * 2.0 ** -22 + 1300 * 2.0 ** -24
            tol[i, h] = 2 * rel * (p @ np.abs(v[mask[i], h // group])).max() / total + 2.0 ** -24 * np.abs(want[i, h]).max()
    err = np.abs(got - want)
    assert np.all(err <= 1.01 * tol), (err / tol).max()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("hd,nkv,n,nodes,path,paged", [
    (128, 2, 200, 60, [0, 3, 7, 8, 59], False), (64, 3, 61, 200, list(range(1, 200, 3)), True), (128, 1, 0, 256, [255], True),
    (64, 2, 127, 3, [0, 1, 2], False), (128, 1, 64, 130, [0, 1, 64, 65, 66, 128, 129], True), (64, 1, 5, 9, [], True),
    (128, 2, 1, 256, list(range(100, 256)), False)])
def test_accepted_positions_move(torch, st, cache, hd, nkv, n, nodes, path, paged):
    """The accepted positions, in every layer, exactly as held; those before them and other users are left, lengths and pages
    are as after kf_kv_set_len."""
    g = bare_stage(st, nkv, hd, layers=2)
    ctx = n + nodes + 70
    kv = g.kv(2, ctx, 2 * ((ctx + 63) // 64) if paged else None, dtype=cache)
    data = [[(rows(7 * l + u, ctx, nkv, hd), rows(50 + 7 * l + u, ctx, nkv, hd)) for u in range(2)] for l in range(2)]
    for l in range(2):
        for u in range(2):
            kv.write(l, u, 0, *(on(x[:n + nodes] if u else x) for x in data[l][u]))
    kv.set_len(0, ctx)
    kv.accept(1, n, path)
    assert kv.len(1) == n + len(path) and kv.len(0) == ctx
    if paged:
        pages = (ctx + 63) // 64
        assert kv.pages() == (2 * pages, pages - (n + len(path) + 63) // 64)
    at = list(range(n)) + [n + i for i in path]
    for l in range(2):
        check(kv, l, 1, 0, *(held(x, cache)[at] for x in data[l][1]), what=f"layer {l}")
        check(kv, l, 0, 0, *(held(x, cache) for x in data[l][0]), what="other user")
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,path", [(63, list(range(1, 256))), (60, list(range(0, 70)) + list(range(71, 256))),
                                    (62, list(range(4)) + list(range(8, 256)))])
def test_long_paths(torch, st, cache, hd, n, path):
    """Paths over four and five pages, close behind themselves, with their weights."""
    nkv, ctx = 2, n + 256
    g = bare_stage(st, nkv, hd, layers=2)
    kv = g.kv(1, ctx, dtype=cache)
    kv.track()
    data = [(rows(3 + l, ctx, nkv, hd), rows(13 + l, ctx, nkv, hd)) for l in range(2)]
    w = np.random.default_rng(n).uniform(size=(2, nkv, ctx)).astype(np.float32)
    at = list(range(n)) + [n + i for i in path]
    for _ in range(3):
        for l in range(2):
            kv.write(l, 0, 0, *(on(x) for x in data[l]))
            kv.set_weights(l, 0, 0, on(w[l]))
        kv.accept(0, n, path)
        for l in range(2):
            check(kv, l, 0, 0, *(held(x, cache)[at] for x in data[l]), what=f"layer {l}")
            assert np.array_equal(kv.weights(l, 0, 0, len(at)).cpu().numpy(), w[l][:, at])
    g.sync()
    kv.close()
    g.close()


def test_accepting_into_shared_pages(torch, st):
    """A tree on pages that two users share after a fork: the other user's stay as they were."""
    g = bare_stage(st, 1, 64, layers=2)
    kv = g.kv(2, 300, 8)
    k, v = rows(1, 200, 1, 64), rows(2, 200, 1, 64)
    for l in range(2):
        kv.write(l, 0, 0, on(k), on(v))
    kv.set_len(0, 200)
    kv.fork(0, 1)
    kv.accept(1, 100, [3, 50, 70])
    for l in range(2):
        check(kv, l, 0, 0, held(k, "f16"), held(v, "f16"))
        at = list(range(100)) + [103, 150, 170]
        check(kv, l, 1, 0, held(k, "f16")[at], held(v, "f16")[at])
    assert kv.len(0) == 200 and kv.len(1) == 103
    kv.close()
    g.close()


def test_refusals(torch, st):
    g = bare_stage(st, 1, 64, layers=2, group=2)
    kv = g.kv(2, 100, 3, dtype="mxfp4")
    kv.write(0, 0, 0, on(rows(1, 64, 1, 64)), on(rows(2, 64, 1, 64)))
    p, q = torch.full((4,), -1, dtype=torch.int32, device="cuda"), on(rows(3, 4, 2, 64))

    def refused(status, call, *args):
        with pytest.raises(st.KFError) as e:
            call(*args)
        assert e.value.status == status
    refused(3, kv.attend_tree, 0, [0], [61], [4], p, q)      # on no page of the user's
    refused(3, kv.attend_tree, 0, [0], [97], [4], p, q)
    refused(3, kv.attend_tree, 0, [1], [0], [4], p, q)
    refused(1, kv.attend_tree, 0, [0], [-1], [4], p, q)
    refused(1, kv.attend_tree, 0, [2], [1], [4], p, q)
    refused(1, kv.attend_tree, 2, [0], [1], [4], p, q)       # no such layer
    refused(1, kv.attend_tree, 0, [0] * 5, [1] * 5, [1, 1, 1, 1, 0], p, q)
    refused(1, kv.attend_tree, 0, [0, 0], [1, 1], [5, -1], p, q)
    big = torch.zeros((257, 2, 64), device="cuda")
    refused(1, kv.attend_tree, 0, [0], [0], [257], torch.zeros(257, dtype=torch.int32, device="cuda"), big)
    odd = torch.zeros(513, device="cuda")[1:].view(4, 2, 64)
    refused(1, kv.attend_tree, 0, [0], [1], [4], p, odd)
    with pytest.raises(ValueError):
        kv.attend_tree(0, [0], [1], [4], p[:3].contiguous(), q)
    with pytest.raises(ValueError):
        kv.attend_tree(0, [0], [1], [4], p.long(), q)
    with pytest.raises(ValueError):
        kv.attend_tree(0, [0], [1, 2], [4], p, q)
    kv.attend_tree(0, [1], [0], [0], p[:0], q[:0])           # a tree without tokens
    refused(3, kv.accept, 0, 60, [4])
    refused(3, kv.accept, 0, 90, [10])
    refused(3, kv.accept, 0, 101, [])
    refused(1, kv.accept, 0, -1, [])
    refused(1, kv.accept, 2, 0, [])
    refused(1, kv.accept, 0, 0, [1, 1])
    refused(1, kv.accept, 0, 0, [2, 1])
    refused(1, kv.accept, 0, 0, [-1])
    refused(1, kv.accept, 0, 0, [256])
    assert kv.len(0) == 0 and kv.pages() == (3, 2)
    g.sync()
    kv.close()
    g.close()


def test_captured_and_replayed_on_another_stream(torch, st):
    """A captured draft step (the tokens written, attended to, some accepted) reads what tokens, parents and cache are at each
    replay, among eager calls that use the same workspace."""
    hd, nkv, group, n, m = 128, 2, 4, 3000, 30
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(2, n + m)
    kvs = [[on(rows(10 * i + j, n, nkv, hd)) for j in range(2)] for i in range(2)]
    for u in range(2):
        kv.write(0, u, 0, *kvs[u])
    new = [[on(rows(70 + 2 * i + j, m, nkv, hd)) for j in range(2)] for i in range(3)]
    pars = [torch.tensor(draft(i, m - i) + [-2] * i, dtype=torch.int32, device="cuda") for i in range(3)]
    qs = [on(rows(90 + i, m, nkv * group, hd)) for i in range(3)]
    k, v, p, q = (t.clone() for t in (*new[0], pars[0], qs[0]))
    out = torch.empty_like(q)
    path = [0, 4, 5, 17]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)
    with torch.cuda.stream(side):
        eager = []
        for i in range(3):
            kv.write(0, 1, n, *new[i])
            o = kv.attend_tree(0, [1], [n], [m], pars[i], qs[i])
            kv.accept(1, n, path)
            eager.append((o.clone(), *(t.clone() for t in kv.read(0, 1, n, len(path)))))
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            kv.write(0, 1, n, k, v)
            kv.attend_tree(0, [1], [n], [m], p, q, out=out)
            kv.accept(1, n, path)
        for i in (1, 0, 2, 1):
            for t, x in zip((k, v, p, q), (*new[i], pars[i], qs[i])):
                t.copy_(x)
            graph.replay()
            kv.attend(0, [0], [n], qs[i][:1].contiguous())
            got = (out, *kv.read(0, 1, n, len(path)))
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, eager[i])), i
    g.sync()
    kv.close()
    g.close()
