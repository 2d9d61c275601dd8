"""Log probabilities, entropy and alternatives of logit rows and of hidden rows."""
import ctypes

import numpy as np
import pytest

import synth
from tests.test_gpu_cache import bare_stage
from tests.test_gpu_logits import head_stage

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


@pytest.fixture(scope="module")
def g(st):
    stage = bare_stage(st, 1, 64)
    yield stage
    stage.close()


def reference(z, targets, top):
    """(log probabilities, entropy, ids, their log probabilities) of rows z in 64 bits; NaN and +inf logits are left out."""
    z = np.where(np.isnan(z) | (z == np.inf), -np.inf, z).astype(np.float64)
    rows, vocab = z.shape
    with np.errstate(invalid="ignore", divide="ignore"):
        m = z.max(1, keepdims=True)
        x = np.where(np.isinf(m), -np.inf, z - m)
        e = np.exp(x)
        lse = np.where(np.isinf(m[:, 0]), 0.0, np.log(e.sum(1)))
        lp = x - lse[:, None]
        h = -np.where(e > 0, np.exp(lp) * np.where(e > 0, lp, 0), 0).sum(1)
    n = min(top, vocab)
    order = np.argsort(-z, axis=1, kind="stable")[:, :n]
    best = np.take_along_axis(lp, order, 1)
    ids = np.full((rows, top), -1)
    alt = np.full((rows, top), -np.inf)
    ids[:, :n] = np.where(best > -np.inf, order, -1)
    alt[:, :n] = best
    return lp[np.arange(rows), targets], h, ids, alt


def close(got, want, tol, what):
    got = got.cpu().numpy().astype(np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), what
    err = np.abs(got[fine] - want[fine])
    tol = np.broadcast_to(tol, want.shape)[fine]
    assert np.all(err <= tol), (what, (err / tol).max())


def check(r, z, targets, top, what=""):
    """Tolerances: ln S is off by the relative error of S: 2^-23 of each exponential, 2^-23 |x| of its argument (whose
    mean over the distribution is at most ln V < 14), and 2^-24 for each of the fewer than 70 additions a value passes
    through: 2^-23 (1 + 14 + 35) < 2^-17; a log probability is rounded twice more, 2^-23 of its size.  The entropy adds
    the same relative error of W / S, at most ln V, and 2^-23 of the second moment of x under e^x, below 14^2."""
    lp, h, ids, alt = reference(z, targets, top)
    close(r.logprob, lp, 2.0 ** -17 + 2.0 ** -23 * np.abs(np.where(np.isfinite(lp), lp, 0)), (what, "logprob"))
    close(r.entropy, h, 2.0 ** -17 * 15 + 2.0 ** -23 * 196, (what, "entropy"))
    if top:
        assert np.array_equal(r.top_ids.cpu().numpy(), ids), (what, np.argwhere(r.top_ids.cpu().numpy() != ids)[:5].tolist())
        close(r.top_logprobs, alt, 2.0 ** -17 + 2.0 ** -23 * np.abs(np.where(np.isfinite(alt), alt, 0)), (what, "alternatives"))
    else:
        assert r.top_ids is None and r.top_logprobs is None


@pytest.mark.parametrize("top", [0, 1, 5, 20, 32])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (3, 7, 1), (2, 1000, 0), (4, 2049, 3), (1, 8192, 0), (5, 8193, 4),
                                            (3, 40003, 5), (300, 9000, 0), (2, 262144, 0), (40, 151936, 0)])
def test_rows_of_every_length(torch, g, top, rows, vocab, pad):
    rng = np.random.default_rng(rows * vocab + top)
    z = (rng.normal(size=(rows, vocab)) * 4).astype(np.float32)
    t = rng.integers(0, vocab, rows).astype(np.int32)
    wide = torch.full((rows, vocab + pad), float("nan"), device="cuda")  # what lies between rows is not read
    wide[:, :vocab] = torch.from_numpy(z)
    check(g.logits_logprobs(wide[:, :vocab], torch.from_numpy(t).cuda(), top=top), z, t, top)
    g.sync()


def test_the_largest_vocabulary(torch, g):
    """2^20 logits a row, in as many chunks as a row may have, with the largest values at both ends and in runs of one chunk."""
    n = 1 << 20
    z = (np.random.default_rng(8).normal(size=(2, n)) * 3).astype(np.float32)
    z[0, [0, n - 1]] = 40, 41
    z[1, 8192 * 77:8192 * 77 + 40] = 30
    t = np.array([n - 1, 8192 * 77 + 39], np.int32)
    check(g.logits_logprobs(torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda(), top=32), z, t, 32)
    g.sync()


@pytest.mark.parametrize("top", [6, 7, 32])
@pytest.mark.parametrize("vocab", [2049, 16384, 16385, 60000])
def test_alternatives_spread_over_chunks(torch, g, top, vocab):
    """The largest values all in the first, a middle or the last chunk of 2048, one in each, equal everywhere (as many
    candidates as a workgroup has threads, and more) and fewer left than asked for."""
    rng = np.random.default_rng(vocab + top)
    z = rng.normal(size=(8, vocab)).astype(np.float32)
    z[0, :40] += 20
    z[1, vocab // 2:vocab // 2 + 40] += 20
    z[2, -40:] += 20
    z[3, ::2048] += 20
    z[4] = 1.25
    z[5] = -np.inf
    z[5, rng.permutation(vocab)[:top - 1]] = rng.normal(size=top - 1)
    z[6, 5:] = -np.inf
    z[7, ::100] = 4.5
    t = rng.integers(0, vocab, 8).astype(np.int32)
    check(g.logits_logprobs(torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda(), top=top), z, t, top)
    g.sync()


def test_more_rows_than_one_launch_takes(torch, g):
    z = (np.random.default_rng(3).normal(size=(32770, 33)) * 3).astype(np.float32)
    t = np.arange(32770).astype(np.int32) % 33
    check(g.logits_logprobs(torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda(), top=2), z, t, 2)
    g.sync()


@pytest.mark.parametrize("vocab", [100, 5000, 70001])
def test_masks_ties_and_extremes(torch, st, g, vocab):
    """Rows with nothing left, one value left, the type's lowest value, equal values everywhere or at the border of the
    alternatives, ascending and descending rows, both zeros, and peaks beyond which everything vanishes."""
    rng = np.random.default_rng(vocab)
    top = 20
    z = (rng.normal(size=(14, vocab)) * 3).astype(np.float32)
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, vocab - 1] = -3.5
    z[2] = np.finfo(np.float32).min
    z[3] = np.finfo(np.float32).min
    z[3, 17] = 0
    z[4] = 2.5
    z[5] = np.round(z[5])
    z[6] = np.sort(z[6])
    z[7] = -np.sort(-z[7])
    z[8] = 0.0
    z[8, ::2] = -0.0
    z[9, 50] = 1e30
    z[10, rng.permutation(vocab)[: vocab - 5]] = -np.inf
    z[11] = -1e30 + z[11]
    z[12, : min(vocab, 4096)] = 50.0
    z[13] = np.repeat(rng.normal(size=(vocab + 31) // 32), 32)[:vocab]
    t = rng.integers(0, vocab, 14).astype(np.int32)
    t[1], t[3], t[9] = vocab - 1, 17, 50
    check(g.logits_logprobs(torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda(), top=top), z, t, top)
    g.sync()


def test_nan_infinity_and_bad_targets(torch, st, g):
    z = np.random.default_rng(0).normal(size=(6, 9000)).astype(np.float32)
    z[0, 3], z[1, 8999], z[2] = np.nan, np.inf, np.nan
    t = np.array([5, 8999, 3, -1, 9000, -2], np.int32)
    r = g.logits_logprobs(torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda(), top=3)
    lp, h, ids, alt = reference(z, np.clip(t, 0, 8999), 3)
    assert np.array_equal(r.top_ids.cpu().numpy(), ids)
    close(r.entropy, h, 2.0 ** -13, "entropy")
    got = r.logprob.cpu().numpy()
    assert abs(got[0] - lp[0]) < 1e-4 and np.isnan(got[[1, 2, 4, 5]]).all() and got[3] == 0
    with pytest.raises(st.KFError) as e:
        g.sync()
    assert e.value.status == 1 and "NaN" in e.value.message and "token" in e.value.message
    g.sync()


@pytest.mark.parametrize("io", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [1, 4, 5, 70, 300])
def test_hidden_rows_as_their_logits(torch, st, rows, io):
    """The call's results are those of its logits, whichever path computes them, with rows left as they were behind."""
    shape, _, g = head_stage(st, 320, 40003, 91)
    x = torch.from_numpy(synth.hidden_states(91, synth.STREAM_DECODE_HIDDEN, 0, rows, 320)).to(getattr(torch, io)).cuda()
    t = torch.from_numpy(np.random.default_rng(1).integers(0, 40003, rows).astype(np.int32)).cuda()
    r = g.head_logprobs(x, t, top=7)
    z = g.head_logits(x)
    check(r, z.cpu().numpy(), t.cpu().numpy(), 7)
    again = g.head_logprobs(x, t, top=7)
    assert all(torch.equal(a, b) for a, b in zip(r, again))
    only = g.head_logprobs(x, top=2, entropy=False)
    assert only.logprob is None and only.entropy is None and torch.equal(only.top_ids, r.top_ids[:, :2])
    few = g.head_logprobs(x, t)
    assert few.top_ids is None and torch.equal(few.logprob, r.logprob) and torch.equal(few.entropy, r.entropy)
    g.sync()
    g.close()


def test_bf16_rows_of_any_size(torch, st):
    """Bf16 rows, few and many, from far below eps to the type's largest and with values of every size in a row, against
    64-bit sums over the stored matrix; a row of zeros, and a NaN that stays in its row."""
    shape, head, g = head_stage(st, 320, 5000, 95, lambda h: h["final_norm"].fill(0x3F80))  # gains of one
    x = synth.hidden_states(95, synth.STREAM_DECODE_HIDDEN, 0, 8, 320)
    x[0] *= 1e-37
    x[1] *= 1e30
    x[2] *= np.exp(np.linspace(-25, 0, 320))
    x[3] = 0
    x[5] *= 3e-3
    x[6, 7] = 1e6
    x = torch.from_numpy(x).bfloat16().cuda()
    w = (head["lm_head"].astype(np.uint32) << 16).view(np.float32).astype(np.float16).astype(np.float64)
    xd = x.float().cpu().numpy().astype(np.float64)
    z = xd / np.sqrt((xd * xd).mean(1, keepdims=True) + np.float64(np.float32(shape.rms_eps))) @ w.T
    t = torch.arange(8, dtype=torch.int32, device="cuda")
    for rows in ([0, 1, 2, 3], [4, 5], [6, 7, 2], [0, 1, 2, 3, 4, 5, 6, 7], [7] * 40 + [6, 3, 0, 1]):
        r = g.head_logprobs(x[rows].contiguous(), t[rows].contiguous(), top=5)
        lp, h, ids, alt = reference(z[rows], np.array(rows), 5)
        # a logit is a chain of K / 16 roundings, each 2^-24 of a partial sum of the size of the largest: below 2^-19 of it
        far = 2.0 ** -17 + 2.0 ** -18 * np.abs(z[rows]).max(1)
        close(r.logprob, lp, far + 2.0 ** -23 * np.abs(lp), "logprob")
        close(r.top_logprobs, alt, far[:, None] + 2.0 ** -23 * np.abs(alt), "alternatives")
        close(r.entropy, h, 2.0 ** -17 * 15 + 2.0 ** -23 * 196 + 15 * far, "entropy")
    g.sync()
    x[1, 3] = float("nan")
    for rows in (3, 8):
        r = g.head_logprobs(x[:rows].contiguous(), top=5)
        assert (r.top_ids[1] == -1).all() and (r.top_ids[[0, *range(2, rows)]] >= 0).all()
        with pytest.raises(st.KFError):
            g.sync()
    g.close()


def test_kept_rows(torch, st):
    shape, _, g = head_stage(st, 320, 5000, 92)
    kv = g.kv(3, 10)
    toks = torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    g.decode(kv, [0, 1, 2], [0, 0, 0], tokens=toks, keep=True)
    r = g.head_logprobs(None, toks, top=4, rows=3)
    check(r, g.head_logits(None, rows=3).cpu().numpy(), toks.cpu().numpy(), 4)
    assert torch.equal(r.top_ids[:, 0], g.head_argmax(None, rows=3))
    with pytest.raises(st.KFError) as e:
        g.head_logprobs(None, toks[:2].contiguous(), rows=2)
    assert e.value.status == 4
    g.sync()
    kv.close()
    g.close()


def test_captured_after_a_first_call(torch, st):
    """A first call cannot be captured (it allocates); later ones can, among eager calls that share the workspace or
    make it grow."""
    shape, _, g = head_stage(st, 320, 40003, 93)
    many = torch.from_numpy(synth.hidden_states(93, synth.STREAM_DECODE_HIDDEN, 7, 300, 320)).cuda()
    x = [torch.from_numpy(synth.hidden_states(93, synth.STREAM_DECODE_HIDDEN, i, 4, 320)).cuda() for i in range(2)]
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            with pytest.raises(st.KFError) as e:
                g.head_logprobs(x[0], t, top=5)
            t.add_(0)
        assert e.value.status == 2 and "captured" in e.value.message
        want = [g.head_logprobs(v, t, top=5) for v in x]
        graph = torch.cuda.CUDAGraph()
        held = x[0].clone()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = g.head_logprobs(held, t, top=5)
        for i in (0, 1, 1, 0):
            held.copy_(x[i])
            graph.replay()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
            g.head_logprobs(many, top=5)
            eager = g.head_logprobs(x[1 - i], t, top=5)
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, want[1 - i]))
    g.sync()
    g.close()


def test_refusals(torch, st, g):
    lib, z = g._lib, torch.zeros(2, 50, device="cuda")
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    out, ids = torch.zeros(2, 40, device="cuda"), torch.zeros(2, 40, dtype=torch.int32, device="cuda")

    def call(rows=2, vocab=50, stride=50, logits=p(z), targets=p(ids), lp=p(out), en=p(out), top=0, ti=None, tl=None):
        return lib.kf_logits_logprobs(g.handle, rows, vocab, stride, logits, targets, lp, en, top, ti, tl)
    assert call() == 0
    for bad in (dict(rows=0), dict(vocab=0), dict(stride=49), dict(logits=None), dict(targets=None), dict(lp=None),
                dict(top=33, ti=p(ids), tl=p(out)), dict(top=-1), dict(top=2, ti=p(ids)), dict(top=2, tl=p(out)),
                dict(targets=None, lp=None, en=None)):
        assert call(**bad) == 1, bad
    assert call(vocab=(1 << 20) + 1, stride=(1 << 20) + 1) == 6
    with pytest.raises(st.KFError) as e:
        g.head_logprobs(torch.zeros(1, 64, device="cuda"), top=1)
    assert e.value.status == 4  # no head
    for bad in (z.double(), z[0], z.cpu(), z.t()):
        with pytest.raises((TypeError, ValueError)):
            g.logits_logprobs(bad, top=1)
    with pytest.raises(TypeError):
        g.logits_logprobs(z, torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        g.logits_logprobs(z, torch.zeros(3, dtype=torch.int32, device="cuda"))
    g.sync()


def test_a_beam_search_over_shared_4bit_pages(torch, st):
    """The operators together: a prompt prefilled once into a 4-bit cache, four beams that share its pages, each step
    one decode, the alternatives of the kept rows, and forks to the best; every beam's score is what scoring its
    tokens afresh, from a cache of its own, gives."""
    shape = synth.SHAPE_TINY
    from tests.helpers import SeededModel
    model = SeededModel(shape, 94)
    g = st.Stage(shape, 0, 2, model.layer, model.head())
    beams, steps = 4, 5
    kv = g.kv(2 * beams, 256, 40, dtype="mxfp4")
    prompt = torch.from_numpy(synth.tokens(94, 0, 90, shape.vocab)).cuda()
    y = g.prefill(kv, 0, 0, tokens=prompt)
    r = g.head_logprobs(y[-1:].contiguous(), top=beams)
    scores, tokens = r.top_logprobs[0].tolist(), [[i] for i in r.top_ids[0].tolist()]
    users, spare = list(range(beams)), list(range(beams, 2 * beams))
    for u in users[1:]:
        kv.fork(0, u)
    for _ in range(steps):
        last = torch.tensor([t[-1] for t in tokens], dtype=torch.int32, device="cuda")
        g.decode(kv, users, [kv.len(u) for u in users], tokens=last, keep=True)
        r = g.head_logprobs(None, top=beams, rows=beams, entropy=False)
        found = sorted(((scores[b] + lp, b, i) for b in range(beams)
                        for lp, i in zip(r.top_logprobs[b].tolist(), r.top_ids[b].tolist())), reverse=True)[:beams]
        for (_, b, _), u in zip(found, spare):
            kv.fork(users[b], u)
        for u in users:
            kv.set_len(u, 0)
        users, spare = spare, users
        scores, tokens = [f[0] for f in found], [tokens[b] + [i] for _, b, i in found]
    assert len({tuple(t) for t in tokens}) == beams
    for score, t in zip(scores, tokens):
        own = g.kv(1, 256, dtype="mxfp4")
        x = [g.prefill(own, 0, 0, tokens=prompt)[-1:]]
        for i, tok in enumerate(t[:-1]):
            x.append(g.decode(own, [0], [90 + i], tokens=torch.tensor([tok], dtype=torch.int32, device="cuda")))
        lp = g.head_logprobs(torch.cat(x), torch.tensor(t, dtype=torch.int32, device="cuda")).logprob.sum().item()
        # a step alone and a step of four keep their activations in fp32 and fp16: up to 1e-2 of a hidden row's largest
        # value (the stage's tolerance), and logits of unit scale follow it
        assert abs(lp - score) < 1e-2 * 4 * (steps + 1), (lp, score)
        own.close()
    for u in users:
        kv.set_len(u, 0)
    assert kv.pages() == (40, 40)
    g.sync()
    kv.close()
    g.close()
