"""The table of rotations of users that evictions have taken far (kf_kv_set_dropped): its rows and its memory."""

import numpy as np
import pytest

import synth
from oracle import stage_oracle as so
from tests.helpers import SeededModel
from tests.test_gpu_attend import on, st, torch  # noqa: F401 (fixtures)
from tests.test_gpu_cache import rows

pytestmark = pytest.mark.gpu

SHAPE = synth.ModelShape(1, 512, 4, 2, 128, 704, 0)


def step_key(g, kv, user, w, seed):
    """Decodes one token: its key as the cache holds it, and in 64 bits, [nkv, hd]."""
    n = kv.len(user)
    x = synth.hidden_states(31, synth.STREAM_DECODE_HIDDEN, seed, 1, SHAPE.hidden)
    g.decode(kv, [user], [n], hidden=on(x))
    xn = so.rms_norm(np.asarray(x, np.float64), w["attn_norm"], SHAPE.rms_eps)
    key = so.rope((xn @ w["wk"].T).reshape(1, -1, SHAPE.head_dim), np.asarray([n + kv.dropped(user)]), SHAPE.rope_theta)
    return kv.read(0, user, n, 1)[0][0].double().cpu().numpy(), key[0]


def test_rotations_past_2_to_32_angles(torch, st):
    """70 million positions of 64 pairs: the table's last rows are there, and their rotations those of the formula."""
    model = SeededModel(SHAPE, 31)
    w = {k: so.bf16_to_f64(v) for k, v in model.layer(0).items()}
    g = st.Stage(SHAPE, 0, 1, model.layer)
    kv = g.kv(2, 100)
    for i, dropped in enumerate((70_000_000, 1_000_003, 0)):
        kv.set_len(1, 0)
        kv.write(0, 1, 0, on(rows(1, 40, 2, 128)), on(rows(2, 40, 2, 128)))
        kv.set_len(1, 40)
        kv.set_dropped(1, dropped)
        got, want = step_key(g, kv, 1, w, i)
        # fp16 operands and keys (2^-10 of the largest), and an angle of 2^27 in 64 bits, off by 2^-25
        assert np.abs(got - want).max() <= 3e-3 * np.abs(want).max(), dropped
    g.sync()
    kv.close()
    g.close()


def test_the_table_takes_no_more_than_its_rows(torch, st):
    """Users that are taken on and on: the cache holds its farthest position's rows, 8 bytes a pair, and a quarter more at most,
    and not the shorter tables before."""
    model = SeededModel(SHAPE, 31)
    w = {k: so.bf16_to_f64(v) for k, v in model.layer(0).items()}
    g = st.Stage(SHAPE, 0, 1, model.layer)
    kv = g.kv(1, 100)
    kv.track()
    start = kv.format()[1]
    held_ = [torch.cuda.mem_get_info()[0]]
    row, far = 64 * 8, 0
    for i in range(60):
        kv.set_len(0, 0)
        kv.set_len(0, 50)
        far = far + 40 + i * i * 100
        kv.set_dropped(0, far)
        kv.evict(0, 0, 40)
        far += 10
        if i % 7 == 0:
            got, want = step_key(g, kv, 0, w, i)
            assert np.abs(got - want).max() <= 3e-3 * np.abs(want).max(), far
        assert kv.format()[1] - start <= row * (1.25 * (far + 100) - 100), i
    # (3.6 GB are rows; the device's allocator keeps blocks of 2 MB)
    held_.append(torch.cuda.mem_get_info()[0])
    assert held_[0] - held_[1] <= row * 1.25 * (far + 100) + (64 << 20)
    g.sync()
    kv.close()
    g.close()


@pytest.mark.parametrize("chunk", [False, True])
def test_captured_steps_outlive_the_table_that_they_read(torch, st, chunk):
    """A step or chunk is captured, the table grows several times, and replays give what they gave."""
    model = SeededModel(SHAPE, 31)
    g = st.Stage(SHAPE, 0, 1, model.layer)
    g.set_flags(st.KF_STAGE_ORDERED)
    kv = g.kv(2, 100)
    n = 20 if chunk else 1
    x = on(synth.hidden_states(31, synth.STREAM_PREFILL_HIDDEN, 0, n, SHAPE.hidden))
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g.set_stream(side)

    def run():
        if chunk:
            g.prefill(kv, 0, 40, hidden=x, out=y, noalloc=True)
        else:
            g.decode(kv, [0], [40], hidden=x, out=y)

    def back():
        kv.set_len(0, 40)
        kv.set_dropped(0, 30)
    with torch.cuda.stream(side):
        kv.write(0, 0, 0, on(rows(1, 40, 2, 128)), on(rows(2, 40, 2, 128)))
        back()
        run()
        want = y.clone(), *(t.clone() for t in kv.read(0, 0, 40, n))
        back()
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run()
        fill = []
        for i, far in enumerate((200, 1000, 30_000, 1_000_000)):
            kv.set_dropped(1, far)
            fill.append(torch.full((1 << 20,), float("nan"), device="cuda"))  # where freed memory would be given again
            back()
            kv.write(0, 0, 40, *[torch.zeros((n, 2, 128), device="cuda")] * 2)
            y.zero_()
            graph.replay()
            got = y, *kv.read(0, 0, 40, n)
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), far
    g.sync()
    kv.close()
    g.close()


def test_tables_grow_beside_a_capture_of_another_stage(torch, st):
    """While one stage's stream is captured, another stage's cache is tracked for the first time, evicted and taken far: its
    allocations leave the capture as it is."""
    model = SeededModel(SHAPE, 31)
    a, b = (st.Stage(SHAPE, 0, 1, model.layer) for _ in range(2))
    b.set_flags(st.KF_STAGE_ORDERED)
    ka, kb = a.kv(1, 100), b.kv(1, 100)
    ka.write(0, 0, 0, on(rows(1, 60, 2, 128)), on(rows(2, 60, 2, 128)))
    ka.set_len(0, 60)
    x = on(synth.hidden_states(31, synth.STREAM_DECODE_HIDDEN, 0, 1, SHAPE.hidden))
    y = torch.empty_like(x)
    want = b.decode(kb, [0], [0], hidden=x).clone()
    kb.set_len(0, 0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    b.set_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.decode(kb, [0], [0], hidden=x, out=y)
        ka.track()
        ka.evict(0, 0, 40)
        ka.set_dropped(0, 5000)
    for _ in range(3):
        y.zero_()
        graph.replay()
        side.synchronize()
        assert torch.equal(y, want)
    assert (ka.len(0), ka.dropped(0)) == (40, 5000)
    a.sync()
    b.sync()
    for t in (ka, kb, a, b):
        t.close()
