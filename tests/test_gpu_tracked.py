"""Attention weights of tracked caches: softmax statistics that are carried from page to page, and what steps add."""
import math

import numpy as np
import pytest

import synth
from oracle import stage_oracle as so
from tests.test_gpu_attend import on, st, torch  # noqa: F401 (fixtures)
from tests.helpers import SeededModel
from tests.test_gpu_cache import bare_stage, rows
from tests.test_gpu_weights import layer64

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


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("shape", [synth.ModelShape(1, 512, 8, 2, 64, 704, 0), synth.ModelShape(1, 512, 8, 2, 128, 704, 0, qk_norm=True),
                                   synth.ModelShape(1, 512, 8, 1, 128, 704, 0)], ids=["hd64", "hd128", "group8"])
@pytest.mark.parametrize("lens", [[700], [6000, 30], [1, 64, 2000, 500]])
def test_a_steps_weights_add_up_to_its_heads(torch, st, cache, shape, lens):
    """Keys that share a large value in one place, whose product with a rounded query is off by the same for all of them (of 11
    bits: up to 0.5% of a head's weights): each head's weights of a step add up to 1 all the same, and those of a prefill chunk's last queries too.

    Both passes take the same products of the same queries, scores off by hd + 4 fp32 roundings each (2^-24 of the sum of
    |products| S, in log2 units) and, where the attention has prepared the queries (MXFP4), by 22 bits of them twice; ln 2 of
    that, with 2^-22 for each exponential, 2^-21 for its argument, and 400 additions along a chain."""
    hd, nkv, group = shape.head_dim, shape.n_kv_heads, shape.n_q_heads // shape.n_kv_heads
    model = SeededModel(shape, 12)
    w = {k: so.bf16_to_f64(v) for k, v in model.layer(0).items()}
    g = st.Stage(shape, 0, 1, model.layer)
    kv = g.kv(4, max(lens) + 40, dtype=cache)
    kv.track(12)
    users = list(range(len(lens)))
    x = synth.hidden_states(12, synth.STREAM_DECODE_HIDDEN, 0, len(lens), shape.hidden)
    none = np.zeros((max(lens) + 1, nkv, hd))
    qs = [layer64(np.asarray(x[u:u + 1], np.float64), w, shape, none, none, n, [n])[1][0] for u, n in enumerate(lens)]

    def bound(q, k):
        S = max((np.abs(k[:, h // group]) @ np.abs(q[h])).max() for h in range(len(q))) * math.log2(math.e) / math.sqrt(hd)
        return group * (math.log(2) * (S * (2 * (hd + 4) * 2.0 ** -24 + 2 * 2.0 ** -22) + 2 * 2.0 ** -21) + 2 * 2.0 ** -22 + 400 * 2.0 ** -24)
    for u, n in enumerate(lens):
        k = rows(u, n, nkv, hd, 0.5)
        for i in range(nkv):
            q = qs[u][i * group:(i + 1) * group]
            at = int(np.abs(q).max(0).argmax())
            k[:, i, at] += np.sign(q[np.abs(q[:, at]).argmax(), at]) * 25 * math.sqrt(hd) / np.abs(q[:, at]).max()  # scores of 25
        kv.write(0, u, 0, on(k), on(rows(9 + u, n, nkv, hd)))
        kv.set_len(u, n)
        kv.set_weights(0, u, 0, torch.full((nkv, n + 1), 0.0, device="cuda"))
    g.decode(kv, users, lens, hidden=on(x))
    for u, n in enumerate(lens):
        got = kv.weights(0, u, 0, n + 1).double().sum(1).cpu().numpy()
        k = kv.read(0, u, 0, n + 1)[0].double().cpu().numpy()
        assert np.all(np.abs(got - group) <= bound(qs[u], k)), (u, got - group, bound(qs[u], k))
    h = synth.hidden_states(12, synth.STREAM_PREFILL_HIDDEN, 0, 20, shape.hidden)
    n = lens[0] + 1
    q = layer64(np.asarray(h, np.float64), w, shape, np.zeros((n + 20, nkv, hd)), np.zeros((n + 20, nkv, hd)), n, list(range(n, n + 20)))[1]
    kv.set_weights(0, 0, 0, torch.full((nkv, n + 20), 0.0, device="cuda"))
    g.prefill(kv, 0, n, hidden=on(h))
    got = kv.weights(0, 0, 0, n + 20).double().sum(1).cpu().numpy()
    k = kv.read(0, 0, 0, n + 20)[0].double().cpu().numpy()
    assert np.all(np.abs(got - 12 * group) <= sum(bound(q[8 + i], k) for i in range(12)))
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
def test_a_chunk_without_allocations_records_no_times(torch, st, cache):
    """kf_stage_prefill_noalloc creates no events, on a tracked cache neither; other tracked calls are timed."""
    shape = synth.SHAPE_TINY
    g = st.Stage(shape, 0, 2, SeededModel(shape, 6).layer)
    kv = g.kv(1, 200, dtype=cache)
    kv.track(8)
    h = on(synth.hidden_states(6, synth.STREAM_PREFILL_HIDDEN, 0, 50, shape.hidden))
    g.profile(True)
    g.prefill(kv, 0, 0, hidden=h, out=torch.empty_like(h), noalloc=True)
    assert g.profile_read() == {}
    g.prefill(kv, 0, 50, hidden=h)
    assert g.profile_read()["attn"][0] == 2
    g.profile(False)
    g.sync()
    kv.close()
    g.close()
