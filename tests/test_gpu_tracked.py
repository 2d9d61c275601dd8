"""Attention weights of tracked caches: softmax statistics that are carried from page to page, and what steps add."""
import math

import numpy as np
import pytest

from tests.test_gpu_attend import on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_cache import bare_stage, rows

pytestmark = pytest.mark.gpu


def added(torch, q, k, lens):
    """What query rows q [rows, nq, hd] over the first lens[b] of positions k [n, nkv, hd] add, [nkv, n], in 64 bits on the GPU,
    and how far that may be off: the bound of tests/test_gpu_weights.py, weight_of."""
    n, nkv, hd = k.shape
    kt = k.transpose(0, 1).contiguous()
    want, tol = (torch.zeros((nkv, n), dtype=torch.float64, device="cuda") for _ in range(2))
    for b, m in enumerate(lens):
        qb = q[b].view(nkv, -1, hd).transpose(1, 2).contiguous()
        p = torch.softmax(torch.matmul(kt[:, :m], qb) / math.sqrt(hd), 1)  # [nkv, m, group]
        S = torch.matmul(kt[:, :m].abs(), qb.abs()).amax(1, keepdim=True) * math.log2(math.e) / math.sqrt(hd)
        ds = S * (2.0 ** -22 + (hd + 4) * 2.0 ** -24)
        want[:, :m] += p.sum(2)
        tol[:, :m] += (p * (2 * math.log(2) * ds + 400 * 2.0 ** -24 + 2 * 2.0 ** -22 + 2.0 ** -20)).sum(2)
    return want, tol


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("io", ["float32", "float16"])
@pytest.mark.parametrize("hd,group,at", [(64, 2, [66000]), (64, 8, [33000 - i for i in range(32)]), (128, 4, [33001] * 5 + [200])])
def test_maxima_that_rise_from_page_to_page(torch, st, cache, io, hd, group, at):
    """Every wave goes over several pages, and each page's scores lie above those of the page before (first KV head), below them
    (second) or on both sides: the running maximum and sum of a column move at each page, or at none."""
    nkv, n = 8, max(at)
    g = bare_stage(st, nkv, hd, group=group)
    kv = g.kv(1, n, dtype=cache)
    kv.track()
    k = rows(1, n, nkv, hd, 0.25)
    k[:, 0, 0] += np.linspace(-8, 8, n, dtype=np.float32)
    k[:, 1, 0] -= np.linspace(-8, 8, n, dtype=np.float32)
    k[:, 2, 0] += np.where(np.arange(n) // 64 % 2, 4, -4)
    q = rows(2, len(at), nkv * group, hd, 0.25)
    q[:, :, 0] = 1.5 * math.sqrt(hd)
    q = on(q, getattr(torch, io))
    kv.write(0, 0, 0, on(k), on(k))
    kv.weigh(0, [0] * len(at), at, q)
    got = kv.weights(0, 0, 0, n).double()
    want, tol = added(torch, q.double(), kv.read(0, 0, 0, n)[0].double(), at)
    tol += 2.0 ** -24 * 300 * want
    assert bool(((got - want).abs() <= tol * 1.01).all()), ((got - want).abs() / tol.clamp_min(1e-30)).max().item()
    kv.close()
    g.close()
