"""Every code under every scale byte that a cache in 8 or 4 bits may hold, read back and attended to."""
import numpy as np
import pytest

import oracle
from oracle import kv_mx
from paper_2609_35140_amd import inputs

pytestmark = pytest.mark.gpu
gu = pytest.importorskip("gpu_util")
from test_gpu_kv_mx import dev_u8, same_values, ua  # noqa: E402,F401

LARGEST = {8: 246, 4: 252}     # scale byte of a block whose largest is just below 2^127


def pool(bits, d, last, numbers_alone=False):
    """(codes, scales) of one kv head, [rows, ..]: a block of 32 codes after the other; in 4 bits every pair of codes in a byte."""
    n = 2 ** bits
    if bits == 8:
        blocks = np.arange(n).reshape(-1, 32)
        if numbers_alone:
            blocks = np.where(blocks % 128 == 127, 0, blocks)
    else:
        pairs = np.arange(256)     # low and high half
        blocks = np.stack([pairs % 16, pairs // 16], 1).reshape(-1, 32)
    scale = np.concatenate([[255], np.arange(27, last + 1)]) if not numbers_alone else np.arange(100, last + 1)
    scales = np.repeat(scale, len(blocks))
    codes = np.tile(blocks, (len(scale), 1))
    more = -len(codes) % (d // 32 * 16)
    codes = np.concatenate([codes, np.zeros((more, 32), dtype=codes.dtype)])
    scales = np.concatenate([scales, np.zeros(more, dtype=scales.dtype)])     # codes 0 with byte 0: as a page never written
    if bits == 4:
        codes = codes[:, 0::2] + 16 * codes[:, 1::2]
    return codes.astype(np.uint8).reshape(-1, d * bits // 8), scales.astype(np.uint8).reshape(-1, d // 32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [(8, 4), (4, 8)])
def test_read(ua, bits, d):
    parts = [pool(b, d, LARGEST[b]) for b in bits]
    rows = max(len(c) for c, _ in parts)
    P = rows // 16
    parts = [np.concatenate([x, np.zeros((rows - len(x), x.shape[1]), dtype=np.uint8)]).reshape(P, 1, 16, -1)
             for pair in parts for x in pair]
    table = np.arange(P, dtype=np.int32)[None]
    seq, pos = np.zeros(rows, dtype=np.int32), np.arange(rows, dtype=np.int32)
    got = ua.kv_read_mx(*(dev_u8(x) for x in parts), gu.dev_i32(table), gu.dev_i32(seq), gu.dev_i32(pos))
    want = oracle.mx_read(parts, *bits, table, seq, pos)
    for g, w in zip(got, want):
        assert same_values(gu.host_bits(g), w)


@pytest.mark.parametrize("d,hq", [(64, 3), (128, 3), (128, 20)])
@pytest.mark.parametrize("bits", [(8, 8), (4, 4), (8, 4), (4, 8)])
def test_decode(ua, bits, d, hq):
    """All codes in keys (scales near 1) and in values (scales up to the largest): the bf16 decode's bits over the oracle's values."""
    (kc, ks), (vc, vs) = pool(bits[0], d, 134, numbers_alone=True), pool(bits[1], d, LARGEST[bits[1]] - 8, numbers_alone=True)
    n = 2560
    parts = [np.concatenate([x] * (n // len(x) + 1))[:n].reshape(n // 16, 1, 16, -1) for x in (kc, ks, vc, vs)]
    values = [oracle.to_bf16_bits(kv_mx.values(parts[i], parts[i + 1], b)) for i, b in ((0, bits[0]), (2, bits[1]))]
    table = gu.dev_i32(np.arange(n // 16)[None])
    q = gu.dev(inputs.normal_bf16((1, hq, d), 1.0, 660))
    for most in (256, 1300, n):    # one chunk, chunks folded in LDS (not in two blocks of heads of 128), and merged
        lens, cache = gu.dev_i32([most]), [dev_u8(x) for x in parts]
        out, lse = ua.decode_mx(q, *cache, table, lens, most, softmax_scale=2.0 ** -14, return_lse=True)
        want, wlse = ua.decode(q, *(gu.dev(v) for v in values), table, lens, most, softmax_scale=2.0 ** -14, return_lse=True)
        assert np.array_equal(gu.host_bits(out), gu.host_bits(want))
        assert np.array_equal(lse.cpu().numpy().view(np.uint32), wlse.cpu().numpy().view(np.uint32))
        assert np.all(np.isfinite(gu.host_f64(out)))
