"""What an MXFP4 cache keeps beside its pages, and what is said of values that do not fit."""
import pytest

import synth
from tests.helpers import SeededModel
from tests.test_gpu_cache import bare_stage, rows

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


@pytest.mark.parametrize("pages", [40, None, 30000])
def test_prefill_pages_of_what_a_user_can_hold(torch, st, pages):
    """The fp16 pages that prefill works on are as many as one user can hold: the pool, or max_ctx where that is less."""
    nkv, hd, layers, ctx = 2, 128, 3, 1 << 20
    g = bare_stage(st, nkv, hd, layers)
    a, b = g.kv(1, ctx, pages), g.kv(1, ctx, pages, dtype="mxfp4")
    held, most = pages or ctx // 64, min(pages or ctx // 64, ctx // 64)
    values = 64 * nkv * hd  # of K (or V) of a page
    appended = 4 * 2 * values * 2 + 4 * (ctx // 64) * 4  # a decode step's new positions, and their table
    assert b.format()[1] - a.format()[1] == layers * held * values * 2 * (35 / 64 - 2) + appended + most * values * 4
    a.close()
    b.close()
    g.close()


def test_prefill_up_to_the_pools_last_page(torch, st):
    """A user that takes a small pool's every page, in chunks, under a far larger max_ctx: as in a cache of its own size."""
    shape = synth.SHAPE_TINY
    g = st.Stage(shape, 0, 2, SeededModel(shape, 97).layer)
    small, own = g.kv(2, 1 << 18, 5, dtype="mxfp4"), g.kv(1, 320, dtype="mxfp4")
    small.set_len(1, 64)
    small.set_len(0, 64)
    small.set_len(1, 0)  # user 0's pages are not the pool's first ones in order
    small.set_len(0, 0)
    at = 0
    for i, n in enumerate((100, 1, 219)):
        h = torch.from_numpy(synth.hidden_states(97, synth.STREAM_PREFILL_HIDDEN, i, n, shape.hidden)).cuda()
        assert torch.equal(g.prefill(small, 0, at, hidden=h), g.prefill(own, 0, at, hidden=h))
        at += n
    assert small.pages() == (5, 0)
    for l in (0, 1):
        assert all(torch.equal(x, y) for x, y in zip(small.read(l, 0, 0, at), own.read(l, 0, 0, at)))
    g.sync()
    for kv in (small, own):
        kv.close()
    g.close()


def test_what_a_4bit_cache_stored_is_said(torch, st):
    """The range error says what a value became: an infinity, and in an MXFP4 cache 49152 or, a NaN, 0."""
    g = bare_stage(st, 1, 64)
    kv = g.kv(1, 64, dtype="mxfp4")
    k = torch.from_numpy(rows(1, 1, 1, 64)).cuda()
    k[0, 0, 3] = float("nan")
    kv.write(0, 0, 0, k, k)
    with pytest.raises(st.KFError) as e:
        g.sync()
    assert e.value.status == 3 and "49152" in e.value.message and "NaN" in e.value.message
    kv.close()
    g.close()
