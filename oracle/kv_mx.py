"""KV cache in 8 or 4 bits -- TEST INFRASTRUCTURE ONLY (CPU oracle).

The format by its definition: blocks of 32 elements with one power of two as their
scale and one code an element, the code of the nearest value among all that a code can
stand for (ties to the even code).  Written with a search over the list of values, in
float64, where every number that occurs is exact; shares nothing with the GPU kernels.
"""
from __future__ import annotations

import numpy as np

from .attention import bf16_to_f64, to_bf16_bits
from .kv_cache import kv_write

BLOCK = 32
LEAST = -100          # exponent of the smallest scale that a write makes
NAN_SCALE = 255       # scale byte of a block that reads as NaN
TOO_LARGE = 2.0 ** 127


def code_values(bits: int) -> np.ndarray:
    """The value of every code: sign, then exponent and mantissa bits (8: 4 and 3, 4: 2 and 1), without the scale."""
    exponent, mantissa = {8: (4, 3), 4: (2, 1)}[bits]
    bias = 2 ** (exponent - 1) - 1
    values = []
    for code in range(2 ** bits):
        field, m = code >> mantissa & 2 ** exponent - 1, code & 2 ** mantissa - 1
        v = m / 2 ** mantissa * 2.0 ** (1 - bias) if field == 0 else (1 + m / 2 ** mantissa) * 2.0 ** (field - bias)
        values.append(-v if code >> bits - 1 else v)
    values = np.array(values)
    if bits == 8:
        values[[0x7F, 0xFF]] = np.nan   # the one pattern of E4M3 that is no number
    return values


def quantise(rows: np.ndarray, bits: int):
    """bf16 bits [..., d] -> (codes [..., d * bits / 8], scale bytes [..., d / 32]), uint8."""
    x = bf16_to_f64(rows).reshape(-1, BLOCK)
    grid = code_values(bits)[: 2 ** (bits - 1)]
    grid = grid[np.isfinite(grid)]      # ascending magnitudes; a code without sign is its place
    most = grid[-1]
    with np.errstate(invalid="ignore"):
        big = np.max(np.abs(x), axis=1)
        bad = ~(big < TOO_LARGE)
    exps = np.arange(LEAST, 128)
    enough = np.where(bad, 0.0, big)[:, None] <= most * 2.0 ** exps[None]
    e = exps[np.argmax(enough, axis=1)]
    y = np.where(bad[:, None], 0.0, x) / 2.0 ** e[:, None].astype(np.float64)
    code = np.zeros(y.shape, dtype=np.int64)
    mag = np.abs(y)
    for i in range(1, len(grid)):       # past the middle between two values, or on it where the upper code is even
        middle = (grid[i - 1] + grid[i]) / 2
        code = np.where((mag > middle) | ((mag == middle) & (i % 2 == 0)), i, code)
    negative = (np.ascontiguousarray(rows).reshape(-1, BLOCK) >> 15 == 1) & ~bad[:, None]
    code = np.where(negative, code + 2 ** (bits - 1), code)
    scale = np.where(bad, NAN_SCALE, e + 127).astype(np.uint8)
    lead = rows.shape[:-1]
    if bits == 4:
        code = code[:, 0::2] + 16 * code[:, 1::2]
    return code.astype(np.uint8).reshape(*lead, -1), scale.reshape(*lead, -1)


def values(codes: np.ndarray, scales: np.ndarray, bits: int) -> np.ndarray:
    """What codes and scale bytes stand for, float64 [..., d]."""
    if bits == 4:
        codes = np.stack([codes & 15, codes >> 4], axis=-1).reshape(*codes.shape[:-1], -1)
    v = code_values(bits)[codes].reshape(*scales.shape, BLOCK)
    scale = np.where(scales == NAN_SCALE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * scale[..., None]).reshape(codes.shape)


def mx_round(rows: np.ndarray, bits: int) -> np.ndarray:
    """bf16 bits [..., d] -> the bf16 bits that a cache of `bits` bits gives back."""
    return to_bf16_bits(values(*quantise(rows, bits), bits))


def mx_write(cache, k_new, v_new, k_bits, v_bits, block_table, seq_idx, positions):
    """(k_codes, k_scales, v_codes, v_scales) after the write (copies)."""
    (kc, ks), (vc, vs) = quantise(k_new, k_bits), quantise(v_new, v_bits)
    codes = [kv_write(cache[i], cache[i], new, new, block_table, seq_idx, positions)[0]
             for i, new in ((0, kc), (1, ks), (2, vc), (3, vs))]
    return tuple(codes)


def mx_read(cache, k_bits, v_bits, block_table, seq_idx, positions):
    """(k, v) bf16 bits [N, Hkv, d] of the tokens' rows; zeros for a token without a place."""
    page = cache[0].shape[2]
    out = []
    for codes, scales, bits in ((cache[0], cache[1], k_bits), (cache[2], cache[3], v_bits)):
        rows = np.zeros((len(positions), codes.shape[1], scales.shape[3] * BLOCK), dtype=np.uint16)
        for n, (s, pos) in enumerate(zip(seq_idx, positions)):
            if pos < 0 or not 0 <= s < block_table.shape[0] or pos // page >= block_table.shape[1]:
                continue
            phys = block_table[s, pos // page]
            if 0 <= phys < codes.shape[0]:
                rows[n] = to_bf16_bits(values(codes[phys, :, pos % page], scales[phys, :, pos % page], bits))
        out.append(rows)
    return tuple(out)
