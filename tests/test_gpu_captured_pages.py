"""Pages that a paged cache lends while a graph is captured: eager calls and later replays agree on whose they are."""
import numpy as np
import pytest

from tests.test_gpu_cache import bare_stage, check, held, rows

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


HD, NKV = 64, 2


class Bench:
    """A two-layer stage on a stream of its own, and a paged cache of four users."""

    def __init__(self, torch, st, dtype, pages=12):
        self.torch, self.dtype = torch, dtype
        self.g = bare_stage(st, NKV, HD, layers=2)
        self.kv = self.g.kv(4, 320, pages, dtype=dtype)
        self.side = torch.cuda.Stream()
        torch.cuda.synchronize()
        self.g.set_stream(self.side)

    def data(self, seed, n):
        """Rows on the device, and what the cache holds of them."""
        x = [rows(seed + i, n, NKV, HD) for i in range(2)]
        return [self.torch.from_numpy(t).cuda() for t in x], [held(t, self.dtype) for t in x]

    def capture(self, work):
        graph = self.torch.cuda.CUDAGraph()
        with self.torch.cuda.graph(graph, stream=self.side):
            work()
            self.pad.add_(0)  # a graph has a node whatever the calls record
        return graph

    def __enter__(self):
        self.scope = self.torch.cuda.stream(self.side)
        self.scope.__enter__()
        self.pad = self.torch.zeros(1, device="cuda")
        return self

    def __exit__(self, *e):
        self.side.synchronize()
        self.scope.__exit__(*e)
        if e[0] is None:
            self.g.sync()
        self.kv.close()
        self.g.close()


@pytest.mark.parametrize("dtype", ["f16", "mxfp4"])
@pytest.mark.parametrize("by", ["write", "set_len"])
def test_eager_calls_before_the_first_replay_find_the_pages(torch, st, dtype, by):
    """A capture that lends user 0 its pages and is never, or only later, replayed: writes, reads, attention, copies and
    forks find them, and the other users' pages stay as they are."""
    with Bench(torch, st, dtype) as b:
        kv = b.kv
        (other, other_held), (mine, mine_held), (late, late_held) = b.data(1, 150), b.data(3, 100), b.data(5, 100)
        for l in (0, 1):
            kv.write(l, 1, 0, *other)
        kv.set_len(1, 150)
        b.side.synchronize()
        graph = b.capture(lambda: kv.write(0, 0, 0, *late) if by == "write" else kv.set_len(0, 100))
        assert kv.pages() == (12, 7)
        for l in (0, 1):
            kv.write(l, 0, 0, *mine)
        kv.set_len(0, 100)
        for l in (0, 1):
            check(kv, l, 1, 0, *other_held, what="another user's")
            check(kv, l, 0, 0, *mine_held)
        kv.fork(0, 2)
        kv.copy(kv, 0, 3, 0, 100)
        q = torch.from_numpy(rows(9, 3, NKV, HD)).cuda()
        a = kv.attend(1, [0, 2, 3], [100] * 3, q[:1].repeat(3, 1, 1))
        assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])
        for _ in range(2):
            graph.replay()
            b.side.synchronize()
            check(kv, 1, 1, 0, *other_held, what="another user's, after a replay")
            check(kv, 1, 0, 0, *mine_held)
            check(kv, 0, 3, 0, *mine_held)
            check(kv, 0, 0, 0, *(late_held if by == "write" else mine_held))


@pytest.mark.parametrize("dtype", ["f16", "mxfp4"])
def test_a_replay_leaves_later_pages_in_place(torch, st, dtype):
    """A page lent in a capture, then shared and copied for its first user: a replay does not put the old page back, so
    that neither its own writes nor later eager ones reach the other user; nor after pages were given back and lent anew."""
    with Bench(torch, st, dtype) as b:
        kv = b.kv
        (base, base_held), (one, one_held), (two, two_held), (three, three_held) = (b.data(10 * i, n) for i, n in
                                                                                   enumerate((128, 2, 2, 2)))
        for l in (0, 1):
            kv.write(l, 0, 0, *base)
        kv.set_len(0, 128)
        b.side.synchronize()
        graph = b.capture(lambda: kv.write(0, 0, 128, *one))  # lends the third page
        graph.replay()
        kv.set_len(0, 130)
        check(kv, 0, 0, 0, *(np.concatenate([x, y]) for x, y in zip(base_held, one_held)))
        kv.fork(0, 1)
        kv.write(0, 0, 128, *two)  # user 0 gets a copy of the third page
        assert kv.pages() == (12, 8)
        check(kv, 0, 1, 128, *one_held)
        for _ in range(3):
            graph.replay()
            b.side.synchronize()
            check(kv, 0, 0, 128, *one_held)
            check(kv, 0, 1, 128, *one_held)
            kv.write(0, 0, 128, *three)
            check(kv, 0, 0, 128, *three_held)
            check(kv, 0, 1, 128, *one_held, what="the other user's page")
            kv.write(0, 1, 128, *two)  # its own page by now
            check(kv, 0, 0, 128, *three_held)
            check(kv, 0, 1, 128, *two_held)
            kv.write(0, 1, 128, *one)
        # given back and lent anew, to others first
        kv.set_len(0, 0)
        for l in (0, 1):
            kv.write(l, 2, 0, *base)
            kv.write(l, 0, 0, *base)
        kv.write(0, 0, 128, *two)
        kv.write(0, 2, 128, *two)
        graph.replay()
        b.side.synchronize()
        check(kv, 0, 0, 128, *one_held)
        check(kv, 0, 2, 0, *(np.concatenate([x, y]) for x, y in zip(base_held, two_held)))
        check(kv, 0, 1, 128, *one_held)


@pytest.mark.parametrize("dtype", ["f16", "mxfp4"])
def test_a_second_capture_finds_what_the_first_lent(torch, st, dtype):
    """Pages lent in one graph and used in a second that is replayed alone, first; and lent twice for one place."""
    with Bench(torch, st, dtype) as b:
        kv = b.kv
        (other, other_held), (x, x_held), (y, y_held) = b.data(1, 64), b.data(3, 70), b.data(5, 70)
        kv.write(0, 1, 0, *other)  # holds the pool's first page, which an unwritten table entry names
        b.side.synchronize()
        first = b.capture(lambda: kv.write(0, 0, 0, *x))
        out = [torch.empty(70, NKV, HD, device="cuda") for _ in range(2)]

        def use():
            kv.write(0, 0, 0, *y)
            for o, r in zip(out, kv.read(0, 0, 0, 70)):
                o.copy_(r)
        second = b.capture(use)
        for _ in range(3):
            second.replay()
            b.side.synchronize()
            assert all(np.array_equal(o.cpu().numpy(), h) for o, h in zip(out, y_held))
        first.replay()
        check(kv, 0, 0, 0, *x_held)
        check(kv, 0, 1, 0, *other_held)
        second.replay()
        check(kv, 0, 0, 0, *y_held)

        def twice():
            kv.write(0, 2, 0, *x)
            kv.set_len(2, 0)
            kv.write(0, 2, 0, *y)
        third = b.capture(twice)
        free = kv.pages()[1]
        third.replay()
        check(kv, 0, 2, 0, *y_held)
        kv.write(0, 2, 0, *x)
        check(kv, 0, 2, 0, *x_held)
        third.replay()
        check(kv, 0, 2, 0, *y_held)
        check(kv, 0, 0, 0, *y_held)
        check(kv, 0, 1, 0, *other_held)
        assert kv.pages()[1] == free
        # forked over: the place's entry is the other user's page now, whatever the third graph lent for it
        kv.set_len(0, 70)
        kv.set_len(2, 0)
        kv.fork(0, 2)
        kv.set_len(2, 0)
        kv.write(0, 2, 0, *x)
        third.replay()
        check(kv, 0, 0, 0, *y_held)
        check(kv, 0, 1, 0, *other_held)
        check(kv, 0, 2, 0, *y_held)


@pytest.mark.parametrize("dtype", ["f16", "mxfp4"])
def test_captured_decode_and_prefill_that_take_pages(torch, st, dtype):
    """Steps and chunks that take pages while they are captured, on a paged cache, give at every replay, and in eager
    calls made before the first one, what they give on a reserved cache; the other users' pages stay as they are."""
    import synth
    from tests.helpers import SeededModel
    shape = synth.SHAPE_TINY
    g = st.Stage(shape, 0, 2, SeededModel(shape, 98).layer)
    g.set_flags(st.KF_STAGE_ORDERED)
    paged, flat = g.kv(4, 320, 14, dtype=dtype), g.kv(4, 320, dtype=dtype)
    side = torch.cuda.Stream()
    h = [torch.from_numpy(synth.hidden_states(98, synth.STREAM_PREFILL_HIDDEN, i, n, shape.hidden)).cuda()
         for i, n in enumerate((64, 64, 100, 2, 128))]
    out = [torch.empty_like(x) for x in h]
    pad = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    g.set_stream(side)

    def chunk(kv):
        return g.prefill(kv, 2, 0, hidden=h[2], out=out[2], noalloc=True)

    def step(kv):
        return g.decode(kv, [0, 1], [64, 64], hidden=h[3], out=out[3])

    with torch.cuda.stream(side):
        for kv in (paged, flat):
            for u in (3, 0, 1):  # user 3 holds the pool's first pages
                g.prefill(kv, u, 0, hidden=h[4] if u == 3 else h[u])
        want = chunk(flat).clone(), step(flat).clone()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            chunk(paged)
            step(paged)
            pad.add_(0)
        assert paged.pages() == (14, 6) and [paged.len(u) for u in range(4)] == [65, 65, 100, 128]
        for u in (0, 1):
            paged.set_len(u, 64)
        paged.set_len(2, 0)
        eager = chunk(paged).clone(), step(paged).clone()
        assert all(torch.equal(a, b) for a, b in zip(eager, want))
        for i in range(3):
            for o in out:
                o.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(out[2], want[0]) and torch.equal(out[3], want[1]), i
            for u in range(4):
                for l in (0, 1):
                    n = flat.len(u)
                    assert all(torch.equal(a, b) for a, b in zip(paged.read(l, u, 0, n), flat.read(l, u, 0, n))), (i, u, l)
            if i == 1:  # moved to other pages, by a fork that goes on writing
                paged.fork(0, 2)
                paged.set_len(2, 0)
                paged.set_len(1, 0)
                g.prefill(paged, 2, 0, hidden=h[2])
                g.prefill(paged, 1, 0, hidden=h[1])
                paged.set_len(1, 65)
    g.sync()
    for kv in (paged, flat):
        kv.close()
    g.close()
