"""MXFP4 caches in 64 bits: what a block of 32 values is stored as (include/kafila_stage.h, kf_kv_create_typed)."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def stored(x) -> np.ndarray:
    """The float64 values that an MXFP4 cache holds for x [..., hd] (finite or infinite float values; NaN gives 0)."""
    with np.errstate(over="ignore"):
        h = np.asarray(x, np.float32).astype(np.float16).astype(np.float64)
    h = np.where(np.isnan(h), 0.0, h)
    b = h.reshape(*h.shape[:-1], h.shape[-1] // BLOCK, BLOCK)
    top = np.abs(b).max(-1, keepdims=True)
    m, e = np.frexp(np.where(np.isinf(top), 2.0 ** 16, top))  # top = m 2^e with m in [0.5, 1)
    e = np.where(m >= 0.875, e + 1, e) - 1 - 2
    e = np.clip(np.where(top == 0, -23, e), -23, 13)
    scale = 2.0 ** e
    a = np.minimum(np.abs(b) / scale, 6.0)
    i = np.searchsorted(MAGNITUDES, a, side="right") - 1  # the element at or below
    up = np.minimum(i + 1, 7)
    low, high = a - MAGNITUDES[i], MAGNITUDES[up] - a
    i = np.where((high < low) | ((high == low) & (up % 2 == 0)), up, i)
    return (np.sign(b) * MAGNITUDES[i] * scale).reshape(h.shape)
