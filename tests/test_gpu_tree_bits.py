"""Attention of drafted trees: the bits that its queries and probabilities keep, for every type of them."""
import math

import numpy as np
import pytest

from tests.test_gpu_attend import EPS, on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_cache import bare_stage, held, rows
from tests.test_gpu_tree import allowed, draft, sees, want_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bfloat16", "float32", "float16"])
@pytest.mark.parametrize("hd,group", [(128, 8), (64, 8), (128, 5), (64, 1)])
@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_two_positions_weigh_as_22_bits_give(torch, st, cache, hd, group, io):
    """A cached position and one token, whose keys have one value each, 1 and -1 at the same place, so that a score is one
    product, and sums of two: what is left is the bits of queries and probabilities.

    Scores are +-s in log2 units with |s| at most 2: off by 2^-22 |s| for the query's two parts (none for one part of bf16)
    and 2^-22 |s| for the factor that takes them there, below 2^-20 together.  The argument of the exponential is the score
    less the reference plus 12, below 16 and rounded once: 2^-21 (what is subtracted and added is rounded the same way for
    both).  A probability is off by ln 2 (2^-20 + 2^-21) for these, 2^-23 for the exponential and 2^-22 for its two parts:
    below 2^-19.2 of itself.  out = (p0 v0 + p1 v1) / (p0 + p1) moves by p0 p1 / (p0 + p1)^2 |v0 - v1| <= |v| / 2 times the
    relative error of p0 / p1, at most twice that: 2^-19.2 |v|.  Ten roundings of sums and the division: 10 2^-24 |v|.
    Together below 2^-18.5 |v|, and half a step of the output's type.  (One part of 11 bits: up to 2^-12 |v|.)"""
    nkv, most = 2, 6.0
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(4, 2, dtype=cache)
    rng = np.random.default_rng(hd + group)
    root = torch.full((4,), -1, dtype=torch.int32, device="cuda")
    worst = 0.0
    for trial in range(32):
        q = np.zeros((4, nkv * group, hd), np.float32)
        want = []
        for u in range(4):
            k, v = np.zeros((2, nkv, hd), np.float32), np.zeros((2, nkv, hd), np.float32)
            v[0] = rng.choice([0.5, 1, 1.5, 2, 3, 4, 6], (nkv, hd)) * rng.choice([-1, 1], (nkv, hd))
            v[:, :, ::32] = 6.0  # the block's largest, so that each value is stored as it is
            v[1] = np.where(v[0] == 6, 6, -v[0])
            for h in range(nkv):
                at = rng.integers(hd)
                k[:, h, at] = 1, -1
                s = rng.uniform(-2, 2, group) * (1 if trial % 2 else 1 / 16) * math.log(2) * math.sqrt(hd)
                q[u, h * group:(h + 1) * group, at] = s
            kv.write(0, u, 0, on(k), on(v))
            assert np.array_equal(held(k, cache), k) and np.array_equal(held(v, cache), v)
            want.append((k.astype(np.float64), v.astype(np.float64)))
        qd = on(q, getattr(torch, io))
        got = kv.attend_tree(0, [0, 1, 2, 3], [1] * 4, [1] * 4, root, qd).float().cpu().numpy().astype(np.float64)
        exact = np.concatenate([want_of(a[None], *kv_, 1, [-1]) for a, kv_ in zip(qd.float().cpu().numpy(), want)])
        half = np.exp2(np.floor(np.log2(np.maximum(np.abs(exact), 1e-30)))) * EPS[io]  # half a step of the output's type
        tol = half * (0 if io == "float32" else 1) + 2.0 ** -18.5 * most
        worst = max(worst, float((np.abs(got - exact) / tol).max()))
    assert worst <= 1, worst
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("io", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("hd,n,m,paged", [(128, 1100, 30, False), (64, 5000, 70, True), (64, 64, 1, False), (128, 20, 3, True)])
def test_infinities_that_a_token_sees(torch, st, io, hd, n, m, paged):
    """An fp16 cache may hold infinities (what did not fit), before the tree and in it.  A value's makes its place of the output
    infinite, with its sign, in every row that sees it, and no other place; a key's of a score of -inf counts for nothing."""
    nkv, group = 2, 4
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(1, n + m, (n + m + 63) // 64 if paged else None)
    k, v = rows(1, n + m, nkv, hd), rows(2, n + m, nkv, hd)
    par = draft(4, m)
    p = torch.tensor(par, dtype=torch.int32, device="cuda")
    q = on(np.abs(rows(3, m, nkv * group, hd, 0.3)) + np.float32(1e-3), getattr(torch, io))
    kv.write(0, 0, 0, on(k), on(v))
    clean = kv.attend_tree(0, [0], [n], [m], p, q).float().cpu().numpy()
    bad = v.copy()
    bad[3, 0, 5], bad[n // 2, 1, 7], bad[n, 1, 40] = np.inf, -np.inf, np.inf  # the last: of the first token
    kv.write(0, 0, 0, on(k), on(bad))
    got = kv.attend_tree(0, [0], [n], [m], p, q).float().cpu().numpy()
    want = clean.copy()
    want[:, :group, 5], want[:, group:, 7] = np.inf, -np.inf
    want[sees(par)[:, 0], group:, 40] = np.inf
    assert np.array_equal(got, want)
    bad = k.copy()
    bad[2, 0, 9] = bad[n - 1, 0, 30] = -np.inf
    kv.write(0, 0, 0, on(bad), on(v))
    got = kv.attend_tree(0, [0], [n], [m], p, q).double().cpu().numpy()
    left = [t for t in range(n + m) if t not in (2, n - 1)]
    qf, kf, vf = q.float().cpu().numpy(), held(k, "f16"), held(v, "f16")
    w = want_of(qf, kf[left], vf[left], n - 2, par)
    assert np.all((np.abs(got - w) <= allowed(qf, kf, vf, w, io))[:, :group])
    assert np.array_equal(got[:, group:], clean[:, group:].astype(np.float64))
    kv.close()
    g.close()
