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
