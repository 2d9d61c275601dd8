"""Attention over caches with given queries: the bits that its queries and probabilities keep, over caches of both types."""
import math

import numpy as np
import pytest

from tests.test_gpu_attend import EPS, allowed, on, want_of
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


@pytest.mark.parametrize("io", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("hd,group", [(128, 8), (64, 8), (128, 5), (64, 1)])
@pytest.mark.parametrize("cache", ["mxfp4", "f16"])
def test_two_keys_weigh_as_22_bits_give(torch, st, cache, hd, group, io):
    """Two positions whose keys have one value each, +-1 at the same place, so that a score is one product, and sums of
    two: what is left is the bits of queries and probabilities, in every place of the head, of 2,000 heads.

    Scores are +-s in log2 units with |s| at most 2: off by 2^-23 |s| for the factor and its product with the query, 2^-22
    |s| for the query's two parts and 2^-24 |s| for their sum, below 2^-20.1.  The argument of the exponential is their
    difference, at most 4 in size, rounded (2^-22), and again with the 12 that is added to it (2^-20): below 2^-19.4.  A
    probability is off by ln 2 (2^-20.1 + 2^-19.4) for these, 2^-23 for the exponential and 2^-22 for its two parts: below
    2^-18.9 of itself.  out = (p0 v0 + p1 v1) / (p0 + p1) moves by p0 p1 / (p0 + p1)^2 |v0 - v1| <= |v| / 2 times the
    relative error of p0 / p1, at most twice that: 2^-18.9 |v|.  Ten roundings of sums and the division: 10 2^-24 |v|.
    Together below 2^-18.5 |v|, and half a step of the output's type.  (One part of 11 bits: up to 2^-12 |v|; two of 8:
    2^-17 |v|.)"""
    nkv, most = 2, 6.0
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(4, 2, dtype=cache)
    rng = np.random.default_rng(hd + group)
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
                s = rng.uniform(-2, 2, group) * math.log(2) * math.sqrt(hd)
                q[u, h * group:(h + 1) * group, at] = s
            kv.write(0, u, 0, on(k), on(v))
            assert np.array_equal(held(k, cache), k) and np.array_equal(held(v, cache), v)
            want.append((k.astype(np.float64), v.astype(np.float64)))
        qd = on(q, getattr(torch, io))
        got = kv.attend(0, [0, 1, 2, 3], [2] * 4, qd).float().cpu().numpy().astype(np.float64)
        exact = np.stack([want_of(a, *kv_) for a, kv_ in zip(qd.float().cpu().numpy().astype(np.float64), want)])
        half = np.exp2(np.floor(np.log2(np.maximum(np.abs(exact), 1e-30)))) * EPS[io]  # half a step of the output's type
        tol = half * (0 if io == "float32" else 1) + 2.0 ** -18.5 * most
        worst = max(worst, float((np.abs(got - exact) / tol).max()))
    assert worst <= 1, worst
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("scale_q,scale_k", [(1e-6, 1.0), (3e-30, 1e3), (1e6, 1e-2), (3e9, 3e-4), (1e6, 1e-5)])
def test_queries_of_any_size_over_an_fp16_cache(torch, st, scale_q, scale_k):
    """Queries far below and above fp16's range keep their bits, and products of large ones with small keys are finite."""
    hd = 64
    g = bare_stage(st, 1, hd, group=8)
    kv = g.kv(1, 300)
    k, v = rows(1, 300, 1, hd, scale_k), rows(2, 300, 1, hd)
    kv.write(0, 0, 0, on(k), on(v))
    k, v = held(k, "f16"), held(v, "f16")
    q = rows(3, 1, 8, hd, scale_q)
    got = kv.attend(0, [0], [300], on(q))[0].cpu().numpy()
    w = want_of(q[0], k, v)
    # the query is in two parts, as over an MXFP4 cache, and the bound that of one
    assert np.all(np.abs(got - w) <= allowed(q[0], k, v, w, "mxfp4", EPS["float32"]))
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("hd,lens", [(128, (1, 15, 16, 17)), (64, (65, 300, 1031, 0))])
def test_an_infinite_value_or_key_shows_in_its_place_only(torch, st, hd, lens):
    """An fp16 cache may hold infinities (what did not fit).  A value's makes its place of the output infinite, with its
    sign, in every row that reads it, and no other place; a key's of a score of -inf counts for nothing."""
    n = 1100
    g = bare_stage(st, 2, hd, group=4)
    kv = g.kv(4, n)
    k, v = rows(1, n, 2, hd), rows(2, n, 2, hd)
    q = np.abs(rows(3, 4, 8, hd, 0.3))
    for u in range(4):
        kv.write(0, u, 0, on(k), on(v))
    clean = kv.attend(0, [0, 1, 2, 3], lens, on(q)).cpu().numpy()
    bad_v, bad_k = v.copy(), k.copy()
    bad_v[0, 1, 5], bad_v[0, 0, 7] = np.inf, -np.inf
    for u in range(4):
        kv.write(0, u, 0, on(k), on(bad_v))
    got = kv.attend(0, [0, 1, 2, 3], lens, on(q)).cpu().numpy()
    # (behind a row's last position its last key is repeated at probability 0: where position 0 is that, 0 inf is NaN)
    for b, m in enumerate(lens):
        want = clean[b].copy()
        if m > 1:
            want[4:, 5], want[:4, 7] = np.inf, -np.inf
            assert np.array_equal(got[b], want), (b, m)
    bad_k[3, 0, 9] = -np.inf
    for u in range(4):
        kv.write(0, u, 0, on(bad_k), on(v))
    got = kv.attend(0, [0, 1, 2, 3], lens, on(q)).cpu().numpy()
    kk = held(k, "f16")
    kk = np.concatenate([kk[:3], kk[4:]])
    vv = held(v, "f16")
    vv = np.concatenate([vv[:3], vv[4:]])
    for b, m in enumerate(lens):
        if m > 3:
            w = want_of(q[b], kk[:m - 1], vv[:m - 1])
            tol = allowed(q[b], kk[:m - 1], vv[:m - 1], w, "mxfp4", EPS["float32"])
            assert np.all((np.abs(got[b] - w) <= tol)[:4]), (b, m)
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["mxfp4", "f16"])
@pytest.mark.parametrize("n", [3, 700])
def test_an_infinite_query_gives_nan_in_its_head_only(torch, st, cache, n):
    g = bare_stage(st, 2, 128, group=3)
    kv = g.kv(1, n, dtype=cache)
    kv.write(0, 0, 0, on(rows(1, n, 2, 128)), on(rows(2, n, 2, 128)))
    q = on(rows(3, 2, 6, 128))
    clean = kv.attend(0, [0, 0], [n, 2], q)
    q[0, 4, 100], q[1, 0, 0] = float("inf"), -float("inf")
    got = kv.attend(0, [0, 0], [n, 2], q)
    bad = torch.zeros(2, 6, dtype=torch.bool, device="cuda")
    bad[0, 4] = bad[1, 0] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])
    kv.close()
    g.close()
