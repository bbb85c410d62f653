"""Pins of the oracle's format in 8 and 4 bits over all bf16 numbers (no GPU): the least exponent in whole-number arithmetic, the
nearest value by brute force, the place of a code in its byte; and mistakes planted in the oracle, which these pins find."""
import functools
import inspect

import numpy as np
import pytest

import oracle
from oracle import kv_mx

MOST = {8: 448, 4: 6}
FINITE = np.concatenate([np.arange(0x7F00), 0x8000 + np.arange(0x7F00)]).astype(np.uint16)   # below 2^127


def _whole(pattern):
    """A bf16 magnitude as m * 2^p."""
    field, m = int(pattern) >> 7 & 0xFF, int(pattern) & 0x7F
    return (m, -133) if field == 0 else (m + 128, field - 134)


def _least_exponent(pattern, most):
    m, p = _whole(pattern)
    e = -100
    while m << max(0, p - e) > most << max(0, e - p):   # m * 2^p > most * 2^e
        e += 1
    return e


@functools.lru_cache(maxsize=None)
def _scales(bits):
    return np.array([_least_exponent(x & 0x7FFF, MOST[bits]) + 127 for x in FINITE[: 0x7F00]] * 2)


def exponents(quantise, bits):
    """Every number as its block's largest: the scale byte."""
    rows = np.zeros((len(FINITE), 32), dtype=np.uint16)
    rows[:, 5] = FINITE
    _, scales = quantise(rows, bits)
    assert np.array_equal(scales[:, 0], _scales(bits))


def codes(quantise, bits):
    """Every number up to the largest as an element of a block whose scale is 1, in an even and an odd place: the code."""
    v = oracle.bf16_to_f64(FINITE)
    x, v = FINITE[np.abs(v) <= MOST[bits]], v[np.abs(v) <= MOST[bits]]
    grid = oracle.code_values(bits)
    with np.errstate(invalid="ignore"):
        off = np.abs(v[:, None] - grid)                 # exact where a tie is possible
    off[:, np.isnan(grid)] = np.inf
    off[np.signbit(v)[:, None] != np.signbit(grid)] = np.inf   # a code has the sign of its number
    near = off == off.min(1, keepdims=True)
    even = near & (np.arange(len(grid)) % 2 == 0)
    want = np.where(near.sum(1) > 1, np.argmax(even, 1), np.argmax(near, 1))
    largest = oracle.to_bf16_bits(np.array([float(MOST[bits])]))[0]
    for first in (0, 1):                                # each in an even place, and in an odd one
        rows = np.full((-(-(len(x) + first) // 31), 32), largest, dtype=np.uint16)
        at = np.arange(len(x)) + first
        rows[at // 31, at % 31] = x
        got, scales = quantise(rows, bits)
        assert np.all(scales == 127)
        if bits == 4:
            got = np.stack([got & 15, got >> 4], -1).reshape(rows.shape)
        assert np.array_equal(got[at // 31, at % 31], want)


def smallest(quantise, bits):
    """Below the least scale: half a step and less is zero, more than half a step is the step."""
    step = {8: 2.0 ** -109, 4: 2.0 ** -101}[bits]
    x = oracle.to_bf16_bits(np.array([0.5 * step, 0.50390625 * step, step, 1.25 * step] + [0.0] * 28))[None]
    assert list(oracle.bf16_to_f64(oracle.to_bf16_bits(kv_mx.values(*quantise(x, bits), bits)))[0, :4]) == [0, step, step, step]


PINS = (smallest, exponents, codes)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("pin", PINS)
def test_pins(pin, bits):
    pin(kv_mx.quantise, bits)


MISTAKES = {
    "ties to the larger code": ("(mag == middle) & (i % 2 == 0)", "(mag == middle)"),
    "ties to the smaller code": ("(mag == middle) & (i % 2 == 0)", "(mag < 0)"),
    "ties to the odd code": ("i % 2 == 0", "i % 2 == 1"),
    "a scale too large where the largest fits exactly": ("<= most", "< most"),
    "a scale that clips": ("<= most", "<= 2 * most"),
    "a lower floor": ("np.arange(LEAST, 128)", "np.arange(LEAST - 1, 128)"),
    "a higher floor": ("np.arange(LEAST, 128)", "np.arange(LEAST + 1, 128)"),
    "the elements of a pair swapped": ("code[:, 0::2] + 16 * code[:, 1::2]", "16 * code[:, 0::2] + code[:, 1::2]"),
    "no sign": ("np.where(negative, code + 2 ** (bits - 1), code)", "code"),
}


@pytest.mark.parametrize("name", MISTAKES)
@pytest.mark.parametrize("bits", [8, 4])
def test_planted_mistakes_are_found(name, bits):
    if bits == 8 and "pair" in name:
        pytest.skip("one element to a byte")
    right, wrong = MISTAKES[name]
    source = inspect.getsource(kv_mx.quantise)
    assert right in source
    scope = dict(vars(kv_mx))
    exec(source.replace(right, wrong), scope)
    for pin in PINS:
        try:
            pin(scope["quantise"], bits)
        except AssertionError:
            return
    pytest.fail("no pin finds it")
