"""The workspaces of the log probabilities: what a first call leaves for later, captured ones, and what they hold."""
import numpy as np
import pytest

import synth
from tests.test_gpu_cache import bare_stage
from tests.test_gpu_logits import head_stage
from tests.test_gpu_logprobs import check

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


def captured(torch, g, side, call):
    graph = torch.cuda.CUDAGraph()
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = call()
    return graph, out


@pytest.mark.parametrize("vocab,first,later", [(128256, 16, (15, 5, 1, 40)), (151936, 14, (13, 2, 100)), (262144, 8, (7, 4, 9)),
                                               (9000, 1, (300,)), (5000, 60, (59, 1))])
def test_a_call_of_any_rows_prepares_captures_of_any(torch, st, vocab, first, later):
    """Rows take chunks of 2048 or 8192 logits by their number, so that fewer rows may have more chunks: a capture of
    fewer or more rows than the eager call before it, with more alternatives and another vocabulary, finds its
    workspace, and gives the bits of an eager call."""
    g = bare_stage(st, 1, 64)
    rng = np.random.default_rng(vocab)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)
    with torch.cuda.stream(side):
        z = torch.from_numpy((rng.normal(size=(first, vocab)) * 3).astype(np.float32)).cuda()
        g.logits_logprobs(z)  # sums only
        graphs = []
        for rows in later:
            for v in (vocab, vocab - 1001):
                z = (rng.normal(size=(rows, v)) * 3).astype(np.float32)
                t = rng.integers(0, v, rows).astype(np.int32)
                zd, td = torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda()
                graphs.append((z, t, zd, td, *captured(torch, g, side, lambda: g.logits_logprobs(zd, td, top=32))))
        for _ in range(3):
            for z, t, zd, td, graph, out in graphs:
                graph.replay()
                side.synchronize()
                eager = g.logits_logprobs(zd, td, top=32)
                assert all(torch.equal(a, b) for a, b in zip(out, eager)), z.shape
                check(out, z, t, 32, z.shape)
    g.sync()
    g.close()


def used(torch, call):
    """Device bytes that a call leaves allocated outside torch's pools."""
    call()  # torch's own blocks
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    call(True)
    torch.cuda.synchronize()
    return before - torch.cuda.mem_get_info()[0]


def test_many_rows_take_a_bounded_workspace(torch, st):
    """The partial results of 20000 rows of 65536 logits are asked for a part of the rows at a time."""
    g, warm = bare_stage(st, 1, 64), bare_stage(st, 1, 64)
    z = torch.zeros(20000, 65536, device="cuda")
    z[:, 77] = 12
    z[19999, 3] = 13
    t = torch.full((20000,), 77, dtype=torch.int32, device="cuda")
    want = np.log(65535 + np.exp(12.0))
    last = np.log(65534 + np.exp(12.0) + np.exp(13.0))
    r = {}

    def call(own=False):
        r["r"] = (g if own else warm).logits_logprobs(z, t, top=2)
    assert used(torch, call) <= 32 << 20
    r = r["r"]
    lp = r.logprob.cpu().numpy().astype(np.float64)
    assert np.abs(lp[:-1] - (12 - want)).max() < 1e-4 and abs(lp[-1] - (12 - last)) < 1e-4
    ids = r.top_ids.cpu().numpy()
    assert np.all(ids[:-1] == [77, 0]) and list(ids[-1]) == [3, 77]
    for s in (g, warm):
        s.sync()
        s.close()


def test_a_workspace_grows_to_what_a_call_asks_for(torch, st):
    """Twenty rows after four, of a wide row and a small vocabulary (whose logits are a hundredth of the workspace): not
    twice the first call's."""
    hidden, vocab = 8192, 500
    _, _, g = head_stage(st, hidden, vocab, 96)
    x = torch.from_numpy(synth.hidden_states(96, synth.STREAM_DECODE_HIDDEN, 0, 20, hidden)).bfloat16().cuda()
    _, _, warm = head_stage(st, hidden, vocab, 96)
    few, more = (used(torch, lambda own=False, n=n: (g if own else warm).head_logprobs(x[:n])) for n in (4, 20))
    assert 0 < few < 8 << 20 and 0 < more <= few + (2 << 20), (few, more)
    for s in (g, warm):
        s.sync()
        s.close()
