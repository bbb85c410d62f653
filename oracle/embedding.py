"""Embedding lookup and its table's gradient -- TEST INFRASTRUCTURE ONLY (CPU
oracle), in float64 from the exact bf16 inputs.  Shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def embedding_fp64(ids, table, scale=1.0):
    """out[t] = scale * table[ids[t]]; negative ids zeros, ids past the table NaN."""
    ids = np.asarray(ids)
    out = np.zeros((ids.size, table.shape[1]))
    ok = (ids >= 0) & (ids < table.shape[0])
    out[ok] = table[ids[ok]] * float(np.float32(scale))
    out[ids >= table.shape[0]] = np.nan
    return out


def embedding_backward_fp64(dout, ids, vocab, scale=1.0, grad=None):
    """(gradient, term magnitudes, tokens per entry); grad: what the sums are added to."""
    out = np.zeros((vocab, dout.shape[1])) if grad is None else grad.copy()
    mag, count = np.abs(out), np.zeros(vocab, dtype=np.int64)
    k = float(np.float32(scale))
    for t, v in enumerate(np.asarray(ids)):
        if 0 <= v < vocab:
            out[v] += k * dout[t]
            mag[v] += abs(k) * np.abs(dout[t])
            count[v] += 1
    return out, mag, count
