"""Drafted trees through a model's layers, against the stage's own steps over the same tokens."""
import math

import numpy as np
import pytest

import synth
from oracle import stage_oracle as so
from tests.helpers import SeededModel, assert_hidden_close
from tests.test_gpu_attend import on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_tree import draft
from tests.test_gpu_weights import layer64, weight_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["f16", "mxfp4"])
@pytest.mark.parametrize("shape", [synth.ModelShape(2, 512, 8, 2, 64, 1408, 1000), synth.ModelShape(2, 512, 8, 2, 128, 704, 0, qk_norm=True)],
                         ids=["tiny", "hd128"])
def test_a_drafted_path_and_steps_meet(torch, st, cache, shape):
    """Two users of one evicted prompt.  One verifies a tree of drafted tokens layer by layer (projections, norms and MLP in 64
    bits, keys and values written, attention by the tree) and accepts a path; the other takes the path's tokens by decode steps.
    Outputs, weights and lengths agree, the next tokens of both in one batch too, and a further eviction of the first goes on
    from there."""
    cfg, n, keep, m = 91, 200, 120, 14
    hd, nkv, nq = shape.head_dim, shape.n_kv_heads, shape.n_q_heads
    model = SeededModel(shape, cfg)
    w = [{k: so.bf16_to_f64(v) for k, v in model.layer(l).items()} for l in range(2)]
    g = st.Stage(shape, 0, 2, model.layer)
    g.set_flags(st.KF_STAGE_ORDERED)
    kv = g.kv(2, 300, 10, dtype=cache)
    kv.track(16)
    g.prefill(kv, 0, 0, hidden=on(synth.hidden_states(cfg, synth.STREAM_PREFILL_HIDDEN, 0, n, shape.hidden)))
    kv.evict(0, 0, keep, 4, 16)
    kv.fork(0, 1)
    assert kv.dropped(0) == kv.dropped(1) == n - keep

    par = draft(5, m)
    depth, path, j = [], [], m - 1
    for p in par:
        depth.append(0 if p < 0 else depth[p] + 1)
    while j >= 0:
        path.insert(0, j)
        j = par[j]
    assert len(path) > 3 and path != list(range(len(path)))
    parents = torch.tensor(par, dtype=torch.int32, device="cuda")
    tokens = synth.hidden_states(cfg, synth.STREAM_DECODE_HIDDEN, 0, m, shape.hidden)
    rot = np.asarray([n + d for d in depth])
    x, queries = np.asarray(tokens, np.float64), []
    for l in range(2):
        xn = so.rms_norm(x, w[l]["attn_norm"], shape.rms_eps)
        q, k, v = ((xn @ w[l][name].T).reshape(m, -1, hd) for name in ("wq", "wk", "wv"))
        if shape.qk_norm:
            q, k = so.rms_norm(q, w[l]["q_norm"], shape.rms_eps), so.rms_norm(k, w[l]["k_norm"], shape.rms_eps)
        q, k = so.rope(q, rot, shape.rope_theta), so.rope(k, rot, shape.rope_theta)
        kv.write(l, 0, keep, on(k.astype(np.float32)), on(v.astype(np.float32)))
        queries.append(on(q.astype(np.float32)))
        a = kv.attend_tree(l, [0], [keep], [m], parents, queries[-1]).double().cpu().numpy()
        x = x + a.reshape(m, -1) @ w[l]["wo"].T
        x = x + so.mlp_swiglu(so.rms_norm(x, w[l]["mlp_norm"], shape.rms_eps), w[l]["wg"], w[l]["wu"], w[l]["wd"])
    kv.accept(0, keep, path)
    before = [[kv.weights(l, u, 0, keep).double().cpu().numpy() for u in range(2)] for l in range(2)]
    for l in range(2):
        kv.weigh(l, [0] * len(path), [keep + i + 1 for i in range(len(path))], queries[l][path].contiguous())

    steps = []
    for i, t in enumerate(path):
        steps.append(g.decode(kv, [1], [keep + i], hidden=on(tokens[t:t + 1])).double().cpu().numpy())
    assert_hidden_close(x[path], np.concatenate(steps), what="path")
    end = keep + len(path)
    assert kv.len(0) == kv.len(1) == end
    for l in range(2):
        got = [kv.weights(l, u, 0, end).double().cpu().numpy() for u in range(2)]
        assert np.array_equal(before[l][0], before[l][1])
        keys = [kv.read(l, u, 0, end)[0].double().cpu().numpy() for u in range(2)]
        q = queries[l].double().cpu().numpy()
        tol = np.zeros((nkv, end))
        for i, t in enumerate(path):
            # a score moves by a step's query (2^-8 of the sum of |products|, a layer's fp16 operands), and by the path's keys,
            # which a step makes of such operands and 4 bits round by up to a fifth of their largest
            a, _ = weight_of(q[t], keys[1], keep + i + 1)
            S = max((np.abs(keys[1][:, h // (nq // nkv)]) @ np.abs(q[t, h])).max() for h in range(nq)) / math.sqrt(hd)
            off = max((np.abs(keys[0][keep:, h // (nq // nkv)] - keys[1][keep:, h // (nq // nkv)]) @ np.abs(q[t, h])).max()
                      for h in range(nq)) / math.sqrt(hd)
            tol[:, :] += a * math.expm1(2 * (2.0 ** -8 * S + off)) + 1e-5
        assert np.all(np.abs(got[0] - got[1]) <= tol), l
        assert np.all(np.abs(got[0].sum(1) - before[l][0].sum(1) - len(path) * (nq // nkv)) <= 1e-3)
        assert np.all(np.abs(got[1].sum(1) - before[l][1].sum(1) - len(path) * (nq // nkv)) <= 1e-3)

    nxt = synth.hidden_states(cfg, synth.STREAM_DECODE_HIDDEN, 1, 1, shape.hidden)
    both = g.decode(kv, [0, 1], [end, end], hidden=on(np.repeat(nxt, 2, 0))).double().cpu().numpy()
    assert_hidden_close(both[:1], both[1:], what="next token")
    kv.evict(0, 0, 80, 4, 16)
    assert kv.dropped(0) == n - keep + end + 1 - 80
    nxt = synth.hidden_states(cfg, synth.STREAM_DECODE_HIDDEN, 2, 1, shape.hidden)
    got = g.decode(kv, [0], [80], hidden=on(nxt)).double().cpu().numpy()
    x = np.asarray(nxt, np.float64)
    for l in range(2):
        k, v = (t.double().cpu().numpy() for t in kv.read(l, 0, 0, 81))
        x, _, _ = layer64(x, w[l], shape, k, v, 80, [80 + kv.dropped(0)])
    assert_hidden_close(got, x, what="after the second eviction")
    g.sync()
    kv.close()
    g.close()
