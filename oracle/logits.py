"""Logit processing (penalties for repeated tokens, biases, masks), its gradient,
and the gradient of the token log-probability -- TEST INFRASTRUCTURE ONLY (CPU
oracle).

Section 3.1 asks for one deterministic logit processing in both regimes and
names no formulas; these are the usual ones, one entry after another in
float64.  Shares no code with the GPU path.
"""
from __future__ import annotations

import numpy as np


def _history(tokens, history, t, vocab):
    """(entries of the whole range, {entry: times in the response}) of row t, the range clamped to the tokens."""
    n = len(tokens)
    begin = min(max(int(history[t][0]), 0), n)
    end = min(max(int(history[t][2]), begin), n)
    split = min(max(int(history[t][1]), begin), end)
    seen = {int(v) for v in tokens[begin:end] if 0 <= v < vocab}
    count = {}
    for v in tokens[split:end]:
        if 0 <= v < vocab:
            count[int(v)] = count.get(int(v), 0) + 1
    return seen, count


def _allowed(mask, mask_rows, t, vocab):
    """[vocab] truth values, or None where the row has no mask."""
    if mask is None:
        return None
    m = t if mask_rows is None else int(mask_rows[t])
    if not 0 <= m < len(mask):
        return None
    words = np.asarray(mask[m]).astype(np.int64) & 0xFFFFFFFF
    v = np.arange(vocab)
    return (words[v // 32] >> (v % 32) & 1).astype(bool)


def logits_process_fp64(logits, tokens=None, history=None, penalties=None, bias_ids=None, bias_values=None,
                        bias_rows=None, mask=None, mask_rows=None):
    """logits [T, V] float64 -> (processed, term magnitudes)."""
    out, mag = logits.astype(np.float64).copy(), np.abs(logits).astype(np.float64)
    T, V = out.shape
    for t in range(T):
        if history is not None:
            seen, count = _history(tokens, history, t, V)
            rep, freq, pres = (float(p) for p in penalties[t])
            for v in seen:
                out[t, v] = out[t, v] / rep if out[t, v] > 0 else out[t, v] * rep
                mag[t, v] = abs(out[t, v])
            for v, n in count.items():
                out[t, v] -= freq * n + pres
                mag[t, v] += abs(freq * n) + abs(pres)
        if bias_rows is not None:
            lo = min(max(int(bias_rows[t][0]), 0), len(bias_ids))
            hi = min(max(int(bias_rows[t][1]), lo), len(bias_ids))
            for v, b in {int(bias_ids[i]): float(bias_values[i]) for i in range(lo, hi)}.items():
                if 0 <= v < V:
                    out[t, v] += b
                    mag[t, v] += abs(b)
        keep = _allowed(mask, mask_rows, t, V)
        if keep is not None:
            out[t, ~keep] = -np.inf
    return out, mag


def logits_process_backward_fp64(dout, logits, tokens=None, history=None, penalties=None, mask=None, mask_rows=None):
    out = dout.astype(np.float64).copy()
    T, V = out.shape
    for t in range(T):
        if history is not None:
            rep = float(penalties[t][0])
            for v in _history(tokens, history, t, V)[0]:
                out[t, v] = out[t, v] / rep if logits[t, v] > 0 else out[t, v] * rep
        keep = _allowed(mask, mask_rows, t, V)
        if keep is not None:
            out[t, ~keep] = 0.0
    return out


def logprob_backward_fp64(logits, targets, dlogp, inv_temperature=1.0):
    """(gradient, bound of an fp32 evaluation's error before its rounding).

    An exponential exp((x - m) it) evaluated in fp32 has an argument off by at most 3
    roundings of its own size (difference, factor, product) and a result off by 2
    steps; a sum of V such terms in a tree adds at most 64 roundings, the products with
    g and 1 / sum four more: relative 2^-24 (3 |arg| + 80), of the sums their weighted mean.
    """
    it = float(np.float32(inv_temperature))
    out, err = np.zeros(logits.shape), np.zeros(logits.shape)
    for t in range(logits.shape[0]):
        g = float(dlogp[t]) * it
        if g == 0.0:
            continue
        y = int(targets[t])
        x = logits[t].astype(np.float64) * it
        if not 0 <= y < x.size or not np.any(x > -np.inf):
            out[t] = np.nan
            continue
        arg = x - x.max()
        e = np.exp(arg)
        others = e.sum() - e[y] if e[y] < 0.5 * e.sum() else e[:y].sum() + e[y + 1:].sum()
        p = e / (others + e[y])
        size = np.where(np.isfinite(arg), np.abs(arg), 0.0)
        off = 2.0 ** -24 * (3.0 * (size + (p * size).sum()) + 80.0)
        out[t], err[t] = -g * p, abs(g) * p * off
        out[t, y] = g * others / (others + e[y])
        rest = np.delete(e * size, y).sum() / max(others, 1e-300)
        err[t, y] = abs(out[t, y]) * 2.0 ** -24 * (3.0 * (rest + (p * size).sum()) + 160.0)
    return out, err + 2.0 ** -126
