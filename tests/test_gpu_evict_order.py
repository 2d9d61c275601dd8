"""Evictions in place, whose pages are moved side by side: what lies there is read before it is overwritten, or the stage says so."""
import ctypes

import numpy as np
import pytest

from tests.test_gpu_attend import on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_cache import bare_stage, check, held, rows
from tests.test_gpu_weights import evicted, kept_of, some_weights

pytestmark = pytest.mark.gpu


@pytest.fixture
def no_patience(st):
    """Pages that would wait for others give up at once (csrc/kernels.h declares the limit; the mangled name is the C++ ABI's)."""
    limit = ctypes.c_int.in_dll(st.load_library(), "_ZN2kf10keep_waitsE")
    old, limit.value = limit.value, 0
    assert old > 1000
    yield limit
    limit.value = old


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("shared", [False, True])
def test_a_wait_that_ends_without_its_flag_is_told(torch, st, no_patience, cache, shared):
    """Every page but the first waits for the one before it.  None of those is written, keys, values (in place) and weights
    alike, and the stage reports it once; the next eviction is as ever."""
    nkv, n, keep, layers = 2, 1000, 500, 2
    g = bare_stage(st, nkv, 64, layers=layers)
    kv = g.kv(2, n, 16 + 8, dtype=cache)
    kv.track()
    data = [(rows(2 * l, n, nkv, 64), rows(2 * l + 1, n, nkv, 64)) for l in range(layers)]
    w = [some_weights(l, nkv, n) for l in range(layers)]
    for l in range(layers):
        kv.write(l, 0, 0, *(on(x) for x in data[l]))
        kv.set_weights(l, 0, 0, on(w[l]))
    kv.set_len(0, n)
    user = 0
    if shared:  # other pages take the places of all that are written
        kv.fork(0, 1)
        user = 1
    kept = kv.evict(user, user, keep, 0, 0, kept=True).cpu().numpy().astype(np.int64)
    with pytest.raises(st.KFError) as e:
        g.sync()
    assert e.value.status == st.KF_ESTATE and "evictions" in e.value.message
    g.sync()
    for l in range(layers):
        at = np.array([kept_of(w[l][h].tolist(), keep, 0, 0) for h in range(nkv)])
        assert np.array_equal(kept[l], at)
        got = kv.weights(l, user, 0, n).cpu().numpy()
        assert np.array_equal(got[:, :64], np.take_along_axis(w[l], at[:, :64], 1), equal_nan=True)
        assert np.array_equal(got[:, 64:], w[l][:, 64:], equal_nan=True)
        pick = lambda x: np.stack([held(x, cache)[at[h], h] for h in range(nkv)], 1)  # noqa: E731
        check(kv, l, user, 0, *(pick(x)[:64] for x in data[l]), what="first page")
        if not shared:
            check(kv, l, 0, 64, *(held(x, cache)[64:keep] for x in data[l]), what="pages left as they were")
        else:
            check(kv, l, 0, 0, *(held(x, cache) for x in data[l]), what="source")
    no_patience.value = 1 << 17
    for u in {0, user}:
        kv.set_len(u, 0)
    for l in range(layers):
        kv.write(l, 0, 0, *(on(x) for x in data[l]))
        kv.set_weights(l, 0, 0, on(w[l]))
    kv.set_len(0, n)
    kept = kv.evict(0, 0, keep, 0, 0, kept=True)
    evicted(kv, layers, nkv, cache, data, w, 0, 0, keep, 0, 0, kept)
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("hd,nkv,layers,n,keep,first,last", [(128, 8, 4, 12000, 7001, 4, 500), (64, 3, 2, 30011, 20003, 70, 0), (128, 1, 1, 20000, 3, 0, 1)])
@pytest.mark.parametrize("shared", [False, True])
def test_contents_of_more_pages_than_fit_side_by_side(torch, st, cache, hd, nkv, layers, n, keep, first, last, shared):
    """Every key and value of evictions in place whose pages outnumber the workgroups that the GPU holds at once (110 pages of
    32 heads in the first case, of 2048), each position its own: on pages of the user's, and where another user holds them too."""
    g = bare_stage(st, nkv, hd, layers=layers)
    pages = (n + 63) // 64
    kv = g.kv(2, n, pages + (keep + 63) // 64, dtype=cache)
    kv.track()
    r = torch.Generator(device="cuda").manual_seed(n)
    data, w = [], []
    for l in range(layers):
        kv.write(l, 0, 0, *(torch.empty((n, nkv, hd), device="cuda").normal_(generator=r) for _ in range(2)))
        data.append([t.clone() for t in kv.read(l, 0, 0, n)])
        w.append(some_weights(l, nkv, n))
        kv.set_weights(l, 0, 0, on(w[l]))
    kv.set_len(0, n)
    user = 0
    if shared:
        kv.fork(0, 1)
        user = 1
    kept = kv.evict(user, user, keep, first, last, kept=True).long()
    g.sync()
    for l in range(layers):
        assert kept[l].tolist() == [kept_of(w[l][h].tolist(), keep, first, last) for h in range(nkv)]
        at = kept[l].t()  # [keep, nkv]
        for got, x in zip(kv.read(l, user, 0, keep), data[l]):
            assert torch.equal(got, x.gather(0, at[:, :, None].expand(-1, -1, hd)))
        assert np.array_equal(kv.weights(l, user, 0, keep).cpu().numpy(), np.take_along_axis(w[l], kept[l].cpu().numpy(), 1), equal_nan=True)
        if shared:
            assert all(torch.equal(a, b) for a, b in zip(kv.read(l, 0, 0, n), data[l]))
    kv.close()
    g.close()


def test_1024_heads_of_a_million_positions(torch, st):
    """An eviction in place of 2^20 positions in 16 layers of 64 heads, 75 GB in 4 bits: 2^32 threads' work.  One position goes, so
    that every other one moves; some are looked at in the first and last layer."""
    nkv, layers, n = 64, 16, 1 << 20
    g = bare_stage(st, nkv, 64, layers=layers)
    kv = g.kv(1, n, dtype="mxfp4")
    kv.track()
    at = [0, 777, 400_000, n - 500]  # first position of each part that has keys and values
    data = {}
    w = torch.ones((nkv, n), device="cuda")
    gone = [700 + 3 * h for h in range(nkv)]
    w[torch.arange(nkv), torch.tensor(gone)] = 0.5
    for l in range(layers):
        kv.set_weights(l, 0, 0, w)
        if l in (0, layers - 1):
            for p in at:
                data[l, p] = [rows(100 * l + p + i, 500, nkv, 64) for i in range(2)]
                kv.write(l, 0, p, *(on(x) for x in data[l, p]))
            kv.set_weights(l, 0, 0, w)  # (written positions start at 0)
    kv.set_len(0, n)
    kv.evict(0, 0, n - 1)
    for l in (0, layers - 1):
        for p in at[2:]:
            check(kv, l, 0, p - 1, *(held(x, "mxfp4") for x in data[l, p]), what=(l, p))
        check(kv, l, 0, 0, *(held(x, "mxfp4") for x in data[l, 0]), what="before")
        assert kv.weights(l, 0, 0, n - 1).eq(1).all()
    g.sync()
    kv.close()
    g.close()
