"""Residual norm (norm behind a block, gate, scale, residual sum, norm before the
next block) and its gradients -- TEST INFRASTRUCTURE ONLY (CPU oracle).

Section 6 Q3 names the hidden and the fused residual RMSNorm; the formulas are
the usual ones:

  u = x r(x) w_post,  s = h + scale gate u,  y = s r(s) w_pre,  r(a) = 1 / sqrt(mean a^2 + eps)

evaluated in float64 from the exact bf16 inputs.  Every value comes with the sum
of the magnitudes of its terms, which bounds what an fp32 evaluation can be off.
Shares no code with the GPU path.
"""
from __future__ import annotations

import numpy as np


def _r(a: np.ndarray, eps: float) -> np.ndarray:
    return 1.0 / np.sqrt(np.mean(a * a, axis=-1, keepdims=True) + eps)


def residual_norm_fp64(residual, pre=None, x=None, post=None, gate=None, scale=1.0, eps=1e-6):
    """All inputs float64 (exact bf16 values) or None.  Returns (s, y) and the term magnitudes of each."""
    scale, eps = float(np.float32(scale)), float(np.float32(eps))
    s, size = residual, np.abs(residual)
    if x is not None:
        u = x if post is None else x * _r(x, eps) * post
        b = scale * u if gate is None else scale * gate * u
        s, size = s + b, size + np.abs(b)
    y = y_size = None
    if pre is not None:
        y = s * _r(s, eps) * pre
        y_size = size * _r(s, eps) * np.abs(pre)
    return (s, y), (size, y_size)


def residual_norm_backward_fp64(dy, dres, h, pre=None, x=None, post=None, gate=None, scale=1.0, eps=1e-6, block=True):
    """Gradients at the stored h and x: dict of values and dict of term magnitudes, keyed
    dresidual, dx, dpre, dpost, dgate (the gate's in the gate's own shape)."""
    scale, eps = float(np.float32(scale)), float(np.float32(eps))
    H = h.shape[-1]
    val, mag = {}, {}
    ds = np.zeros_like(h) if dres is None else dres.copy()
    m_ds = np.abs(ds)
    if dy is not None:
        r = _r(h, eps)
        n, a = h * r, dy * pre
        val["dpre"], mag["dpre"] = (dy * n).sum(0), np.abs(dy * n).sum(0)
        ds = ds + r * (a - n * (a * n).sum(-1, keepdims=True) / H)
        m_ds = m_ds + r * (np.abs(a) + np.abs(n) * np.abs(a * n).sum(-1, keepdims=True) / H)
    val["dresidual"], mag["dresidual"] = ds, m_ds
    if not block:
        return val, mag
    b, m_b = scale * ds, abs(scale) * m_ds
    if post is not None:
        rx = _r(x, eps)
        m = x * rx
    if gate is not None:
        u = x if post is None else m * post
        d, md = b * u, m_b * np.abs(u)
        val["dgate"], mag["dgate"] = (d, md) if gate.ndim == 2 else (d.sum(0), md.sum(0))
        b, m_b = b * gate, m_b * np.abs(gate)
    if post is not None:
        val["dpost"], mag["dpost"] = (b * m).sum(0), (m_b * np.abs(m)).sum(0)
        c, m_c = b * post, m_b * np.abs(post)
        b = rx * (c - m * (c * m).sum(-1, keepdims=True) / H)
        m_b = rx * (m_c + np.abs(m) * (m_c * np.abs(m)).sum(-1, keepdims=True) / H)
    val["dx"], mag["dx"] = b, m_b
    return val, mag
