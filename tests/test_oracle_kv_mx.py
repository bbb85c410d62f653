"""Pins of the oracle's KV cache in 8 or 4 bits (no GPU): by hand, against torch's own 8-bit type, and by what the
format promises (the smallest scale that clips nothing, the nearest value, reading back exactly)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import kv_mx
from paper_2609_35140_amd import inputs


def bits_of(x):
    return oracle.to_bf16_bits(np.asarray(x, dtype=np.float64))


def block(first, rest=0.0, d=64):
    x = np.full(d, rest)
    x[: len(first)] = first
    return bits_of(x)


def test_code_values_by_hand():
    four = oracle.code_values(4)
    assert list(four) == [0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6] and np.signbit(four[8])
    eight = oracle.code_values(8)
    assert eight[0] == 0 and eight[1] == 2.0 ** -9 and eight[7] == 7 * 2.0 ** -9 and eight[8] == 2.0 ** -6
    assert eight[0x38] == 1.0 and eight[0x7E] == 448 and np.isnan(eight[0x7F]) and eight[0xB9] == -1.125


def test_four_bits_by_hand():
    # largest 6 exactly: scale 1; ties go to the even code: 0.25 -> 0, 0.75 -> 1 (code 2), 2.5 -> 2 (4), 3.5 -> 4 (6), 5 -> 4 (6)
    x = [6, 0.25, 0.75, 1.25, 2.5, 3.5, 5, -5, 0.26, -0.0]
    codes, scales = kv_mx.quantise(block(x), 4)
    low_high = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
    assert list(low_high[:10]) == [7, 0, 2, 2, 4, 6, 6, 14, 1, 8]
    assert scales[0] == 127 and scales[1] == 27        # a block of zeros has the smallest scale
    # a little more than 6 takes the next scale
    _, s = kv_mx.quantise(block([6.0625]), 4)
    assert s[0] == 128
    assert list(oracle.bf16_to_f64(oracle.mx_round(block([6.0625, 1.0]), 4))[:2]) == [6.0, 1.0]


def test_eight_bits_are_torchs():
    """Where the scale is 1, the codes are those of torch's own cast."""
    g = inputs.rng(501)
    x = np.concatenate([g.normal(0, s, 3100) for s in (0.01, 1.0, 60.0)])
    x = np.clip(x, -440, 440).reshape(-1, 31)
    rows = bits_of(np.concatenate([np.full((300, 1), 448.0), x[:300]], axis=1).reshape(-1, 64))
    codes, scales = kv_mx.quantise(rows, 8)
    assert np.all(scales == 127)
    t = torch.from_numpy(oracle.bf16_to_f64(rows)).to(torch.float32).to(torch.float8_e4m3fn)
    assert np.array_equal(t.view(torch.uint8).numpy(), codes)


@pytest.mark.parametrize("bits,most", [(8, 448.0), (4, 6.0)])
def test_promises(bits, most):
    g = inputs.rng(502, bits)
    x = g.normal(0, 1, (400, 64)) * 2.0 ** g.integers(-90, 90, (400, 1))
    rows = bits_of(x)
    v = oracle.bf16_to_f64(rows).reshape(-1, 32)
    codes, scales = kv_mx.quantise(rows, bits)
    big = np.abs(v).max(1)
    scale = 2.0 ** (scales.reshape(-1).astype(np.float64) - 127)
    assert np.all(big <= most * scale) and np.all(big > most * scale / 2)     # smallest scale that clips nothing
    held = kv_mx.values(codes, scales, bits).reshape(-1, 32)
    grid = oracle.code_values(bits)
    grid = grid[np.isfinite(grid)]
    best = np.min(np.abs(v[:, :, None] / scale[:, None, None] - grid), axis=2) * scale[:, None]
    assert np.array_equal(np.abs(held - v), best)                            # the nearest value
    half = {8: 2.0 ** -4, 4: 2.0 ** -2}[bits]
    assert np.all(np.abs(held - v) <= np.maximum(half * np.abs(v), np.min(grid[grid > 0]) / 2 * scale[:, None]))
    once = oracle.mx_round(rows, bits)
    assert np.array_equal(oracle.bf16_to_f64(once).reshape(-1, 32), held)    # bf16 holds every value
    assert np.array_equal(oracle.mx_round(once, bits), once)                 # and rounding again changes nothing


@pytest.mark.parametrize("bits", [8, 4])
def test_blocks_that_are_no_numbers(bits):
    for bad in (np.inf, -np.inf, np.nan, 2.0 ** 127, -1.9 * 2.0 ** 127):
        codes, scales = kv_mx.quantise(block([1.0, bad, -3.0], rest=2.0), bits)
        assert scales[0] == 255 and scales[1] != 255 and np.all(codes[: 4 * bits] == 0)
        back = oracle.bf16_to_f64(oracle.mx_round(block([1.0, bad, -3.0], rest=2.0), bits))
        assert np.all(np.isnan(back[:32])) and np.all(back[32:] == 2.0)
    near = block([1.99 * 2.0 ** 126, -(2.0 ** 126)])
    assert np.all(np.isfinite(oracle.bf16_to_f64(oracle.mx_round(near, bits))))
    # under half of the smallest step nothing is left but the sign
    tiny = oracle.mx_round(block([2.0 ** -112, -(2.0 ** -112), 2.0 ** -133]), bits)
    assert list(tiny[:3]) == [0, 0x8000, 0]


def test_write_and_read_by_place():
    g = inputs.rng(503)
    P, hkv, page, d = 4, 2, 16, 64
    cache = tuple(g.integers(0, 127, (P, hkv, page, w)).astype(np.uint8) for w in (64, 2, 32, 2))
    table = np.array([[3, 1], [0, 9]])
    seq, pos = [0, 0, 1, 1, 0, 2], [0, 20, 3, 17, -1, 0]     # 3: page 9 is none, 4: padding, 5: no such sequence
    rows = inputs.normal_bf16((6, hkv, d), 1.0, 504)
    after = oracle.mx_write(cache, rows, rows, 8, 4, table, seq, pos)
    k, v = oracle.mx_read(after, 8, 4, table, seq, pos)
    assert np.array_equal(k[:3], oracle.mx_round(rows, 8)[:3]) and np.array_equal(v[:3], oracle.mx_round(rows, 4)[:3])
    assert np.all(k[3:] == 0) and np.all(v[3:] == 0)
    for a, b in zip(after, cache):
        same = np.all(a == b, axis=-1)
        same[3, :, 0] = same[1, :, 4] = same[0, :, 3] = True
        assert np.all(same)
