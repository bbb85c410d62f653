"""The KV cache in 8 or 4 bits on the GPU: codes, scales and values exactly as the oracle has them, and a decode that has the
bits of the bf16 decode over the same values (which the other tests hold to the full-sequence rows and to the oracle)."""
import numpy as np
import pytest

import oracle
from oracle import kv_mx
from paper_2609_35140_amd import inputs

pytestmark = pytest.mark.gpu
gu = pytest.importorskip("gpu_util")

BITS = [(8, 8), (4, 4), (8, 4), (4, 8)]


@pytest.fixture(scope="module")
def ua():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35140_amd import uattn
    uattn.lib()
    return uattn


def dev_u8(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.uint8)).cuda()


def host_u8(t):
    return t.cpu().numpy()


def same_values(got, want):
    """Equal bf16 bits; any NaN stands for any other."""
    nan = np.isnan(oracle.bf16_to_f64(want))
    return np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want)) and np.array_equal(np.isnan(oracle.bf16_to_f64(got)), nan)


def rows_of(shape, tag, special=True):
    """bf16 rows with everything that a block may hold: all magnitudes, exact ties, zeros, blocks near the limits, NaN and inf."""
    g = inputs.rng(600, tag)
    x = g.normal(0, 1, shape) * 2.0 ** g.integers(-6, 6, shape[:-1] + (1,))
    b = oracle.to_bf16_bits(x).reshape(-1, 32)
    n = len(b)
    if special and n >= 16:
        at = g.permutation(n)[: n // 4 // 8 * 8 or 8].reshape(8, -1)
        b[at[0]] = g.integers(0, 0x7F00, b[at[0]].shape) | g.integers(0, 2, b[at[0]].shape) << 15        # any exponents
        b[at[1]] = g.integers(0x3F80, 0x4140, b[at[1]].shape)                                            # ties and near ones
        b[at[2]] = g.integers(0, 2, b[at[2]].shape) << 15                                                # zeros of both signs
        b[at[3]] = g.integers(0, 0x0900, b[at[3]].shape)                                                 # under the smallest scale
        b[at[4]] = g.integers(0x7E00, 0x7F00, b[at[4]].shape)                                            # the largest numbers
        b[at[5], 7] = 0x7F80
        b[at[6], 31] = 0xFFC1
        b[at[7], 0] = 0x7F00 + at[7] % 0x80                                                              # 2^127 and more
    return b.reshape(shape).astype(np.uint16)


def test_round_every_number(ua):
    """All bf16 patterns, each as its block's largest and among larger ones."""
    every = np.arange(65536, dtype=np.uint16)
    alone = np.zeros((65536, 64), dtype=np.uint16)
    alone[:, 3] = every
    alone[:, 32:] = every[:, None] ^ (np.arange(32, dtype=np.uint16) & 1) << 15
    exponent = np.clip((every >> 7 & 0xFF).astype(np.int64) + (every % 9), 0, 0xFD)
    alone[:, 5] = (exponent << 7).astype(np.uint16)
    for kb, vb in ((8, 4), (4, 8)):
        k, v = ua.kv_round_mx(gu.dev(alone[:, None]), gu.dev(alone[:, None]), kb, vb)
        assert same_values(gu.host_bits(k)[:, 0], oracle.mx_round(alone, kb))
        assert same_values(gu.host_bits(v)[:, 0], oracle.mx_round(alone, vb))


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("N,hkv,d", [(1, 1, 64), (3, 1, 128), (63, 2, 64), (257, 3, 128), (40, 5, 64), (1000, 8, 128)])
def test_round(ua, bits, N, hkv, d):
    import torch
    k, v = rows_of((N, hkv, d), 1), rows_of((N, hkv, d), 2)
    ko, vo = ua.kv_round_mx(gu.dev(k), gu.dev(v), *bits)
    want = oracle.mx_round(k, bits[0]), oracle.mx_round(v, bits[1])
    assert same_values(gu.host_bits(ko), want[0]) and same_values(gu.host_bits(vo), want[1])
    # inside the projection's rows, in place: the query heads beside them stay
    fused = torch.full((N, 2 + 2 * hkv, d), 3.0, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:2 + hkv], fused[:, 2 + hkv:] = gu.dev(k), gu.dev(v)
    parts = fused[:, 2:2 + hkv], fused[:, 2 + hkv:]
    out = ua.kv_round_mx(*parts, *bits, k_out=parts[0], v_out=parts[1])
    assert out[0].data_ptr() == parts[0].data_ptr()
    assert same_values(gu.host_bits(parts[0]), want[0]) and same_values(gu.host_bits(parts[1]), want[1])
    assert bool((fused[:, :2] == 3.0).all())


def _places(g, N, B, maxp, page, P):
    """A table of distinct pages with two entries that are none, and N tokens: distinct places, padding and places that are none."""
    table = g.permutation(P)[: B * maxp].reshape(B, maxp).astype(np.int32)
    table[-1, -1] = -1
    table[0, -1] = P + 3
    slots = g.choice(B * maxp * page, size=N, replace=False)
    seq, pos = slots // (maxp * page), slots % (maxp * page)
    if N > 8:
        pos[3], seq[5], pos[7], seq[8] = -2, B, maxp * page, -1
    return table, seq.astype(np.int32), pos.astype(np.int32)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("N,hkv,d,page", [(1, 1, 64, 16), (7, 2, 128, 16), (100, 3, 64, 32), (33, 8, 128, 64), (301, 1, 128, 16),
                                          (65, 5, 64, 64)])
def test_write_and_read(ua, bits, N, hkv, d, page):
    import torch
    g = inputs.rng(601, N)
    B, maxp = 3, -(-N // page) + 1
    P = B * maxp + 2
    table, seq, pos = _places(g, N, B, maxp, page, P)
    cache = tuple(g.integers(0, 256, (P, hkv, page, w), dtype=np.uint8)
                  for w in (d * bits[0] // 8, d // 32, d * bits[1] // 8, d // 32))
    k, v = rows_of((N, hkv, d), 3), rows_of((N, hkv, d), 4)
    places = gu.dev_i32(table), gu.dev_i32(seq), gu.dev_i32(pos)
    mine = tuple(dev_u8(c) for c in cache)
    fused = torch.full((N, 1 + 2 * hkv, d), 3.0, dtype=torch.bfloat16, device="cuda")   # rows inside the projection's
    fused[:, 1:1 + hkv], fused[:, 1 + hkv:] = gu.dev(k), gu.dev(v)
    ua.kv_write_mx(fused[:, 1:1 + hkv], fused[:, 1 + hkv:], *places, *mine)
    want = oracle.mx_write(cache, k, v, *bits, table, seq, pos)
    for got, w in zip(mine, want):
        assert np.array_equal(host_u8(got), w)
    rows = oracle.mx_read(want, *bits, table, seq, pos)
    got = ua.kv_read_mx(*mine, *places)
    assert same_values(gu.host_bits(got[0]), rows[0]) and same_values(gu.host_bits(got[1]), rows[1])
    # a token that has a place reads what rounding its row gives
    rk, _ = ua.kv_round_mx(gu.dev(k), gu.dev(v), *bits)
    there = [n for n in range(N) if 0 <= seq[n] < B and 0 <= pos[n] < maxp * page and 0 <= table[seq[n], pos[n] // page] < P]
    assert same_values(gu.host_bits(got[0])[there], gu.host_bits(rk)[there])
    # into rows further apart: what lies between them stays
    wide = torch.full((N, 2 * hkv + 1, d), 5.0, dtype=torch.bfloat16, device="cuda")
    ua.kv_read_mx(*mine, *places, k_out=wide[:, :hkv], v_out=wide[:, hkv + 1:])
    assert same_values(gu.host_bits(wide[:, :hkv]), rows[0]) and same_values(gu.host_bits(wide[:, hkv + 1:]), rows[1])
    assert bool((wide[:, hkv] == 5.0).all())


def _equal(got, want):
    """Equal bf16 numbers on the device; any NaN stands for any other."""
    import torch
    nan = torch.isnan(want)
    return bool(torch.equal(torch.isnan(got), nan) and torch.equal(got.view(torch.int16)[~nan], want.view(torch.int16)[~nan]))


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("N,hkv,d", [(8301, 8, 128), (33331, 8, 128), (100003, 6, 64), (262145, 1, 128)])
def test_rows_larger_than_the_caches(ua, bits, N, hkv, d):
    """Rows of 17 to 77 MB (past the caches in some calls, in others not): those of a small call, repeated; places in any order,
    some tokens without one."""
    import torch
    k, v = gu.dev(rows_of((1009, hkv, d), 5)), gu.dev(rows_of((1009, hkv, d), 6))
    small = ua.kv_round_mx(k, v, *bits)
    assert same_values(gu.host_bits(small[0]), oracle.mx_round(gu.host_bits(k), bits[0]))
    assert same_values(gu.host_bits(small[1]), oracle.mx_round(gu.host_bits(v), bits[1]))
    at = torch.arange(N, device="cuda") % 1009
    k, v = k[at], v[at]
    got = ua.kv_round_mx(k, v, *bits)
    assert _equal(got[0], small[0][at]) and _equal(got[1], small[1][at])
    g = inputs.rng(602, N)
    maxp = N // 64 + 1
    table = g.permutation(maxp).astype(np.int32)[None]
    pos = g.permutation(maxp * 64)[:N].astype(np.int32)
    pos[g.integers(0, N, 50)] = -1
    pos[N - 1] = maxp * 64
    places = gu.dev_i32(table), torch.zeros(N, dtype=torch.int32, device="cuda"), gu.dev_i32(pos)
    cache = ua.mx_cache(maxp, hkv, 64, d, *bits)
    ua.kv_write_mx(k, v, *places, *cache)
    back = ua.kv_read_mx(*cache, *places)
    there = torch.from_numpy((pos >= 0) & (pos < maxp * 64)).cuda()[:, None, None]
    for b, w in zip(back, got):
        assert _equal(b, torch.where(there, w, 0))
    # in place
    ua.kv_round_mx(k, v, *bits, k_out=k, v_out=v)
    assert _equal(k, got[0]) and _equal(v, got[1])


def test_past_32_bits(ua):
    """A pool of 4.6 GB of codes and rows 4.4 GB long: offsets that have no 32-bit number."""
    import torch
    P, hkv, page, d, N = 70001, 8, 64, 128, 2200003
    k = torch.empty((N, hkv, d), dtype=torch.bfloat16, device="cuda")
    tail = gu.dev(rows_of((2048, hkv, d), 7, special=False))
    for lo in (0, N - 2048):
        k[lo:lo + 2048] = tail
    kr, vr = ua.kv_round_mx(k, k, 8, 4)
    wk, wv = ua.kv_round_mx(tail, tail, 8, 4)
    for lo in (0, N - 2048):
        assert torch.equal(kr[lo:lo + 2048], wk) and torch.equal(vr[lo:lo + 2048], wv)
    del kr, vr
    big, small = ua.mx_cache(P, hkv, page, d, 8, 4), ua.mx_cache(32, hkv, page, d, 8, 4)
    i32 = dict(dtype=torch.int32, device="cuda")
    high = torch.arange(P - 32, P, **i32)[None]
    low = torch.arange(32, **i32)[None]
    # padding for all rows but the last ones, which go to the last pages
    pos = torch.full((N,), -1, **i32)
    pos[N - 2048:] = torch.arange(2048, **i32)
    zero = torch.zeros(N, **i32)
    ua.kv_write_mx(k, k, high, zero, pos, *big)
    ua.kv_write_mx(tail, tail, low, zero[:2048], pos[N - 2048:], *small)
    for b, s in zip(big, small):
        assert torch.equal(b[P - 32:], s) and not bool(b[:P - 32].any())
    rk, rv = ua.kv_read_mx(*big, high, zero, pos, k_out=k, v_out=torch.empty_like(k))
    assert torch.equal(rk[N - 2048:], wk) and torch.equal(rv[N - 2048:], wv) and not bool(rk[:N - 2048].any())
    q = gu.dev(inputs.normal_bf16((1, 16, d), 1.0, 630))
    n = torch.tensor([2048], **i32)
    assert torch.equal(ua.decode_mx(q, *big, high, n, 2048), ua.decode_mx(q, *small, low, n, 2048))
    wide = torch.full((1, 64), -1, **i32)
    wide[:, :32] = high
    assert torch.equal(ua.decode_mx(q, *big, wide, n, 4096), ua.decode_mx(q, *small, low, n, 2048))


def test_read_without_a_table(ua):
    """No sequences, no table columns, no pages: zeros."""
    import torch
    i32 = dict(dtype=torch.int32, device="cuda")
    seq, pos = torch.zeros(5, **i32), torch.arange(5, **i32)
    for P, B, maxp in ((4, 0, 2), (4, 2, 0), (0, 2, 2)):
        k, v = ua.kv_read_mx(*ua.mx_cache(P, 2, 16, 64, 8, 4), torch.zeros((B, maxp), **i32), seq, pos)
        assert k.shape == (5, 2, 64) and not k.any() and not v.any()
    k, _ = ua.kv_read_mx(*ua.mx_cache(4, 2, 16, 64), torch.zeros((2, 2), **i32), seq[:0], pos[:0])
    assert k.shape == (0, 2, 64)
    assert ua.kv_round_mx(k, k.clone(), 4, 4)[0].shape == (0, 2, 64)


class Cache:
    """Sequences of given lengths in a cache of both kinds: codes, and the bf16 numbers they stand for; NaN in every place that
    no position has."""

    def __init__(self, lens, hkv, d, page, bits, tag, slack=2, special=False, sigma=1.0):
        g = inputs.rng(610, tag)
        self.lens, self.bits, self.page = lens, bits, page
        used = [-(-n // page) for n in lens]
        P = sum(used) + 3
        maxp = max(used) + slack
        order = g.permutation(P)
        self.table = np.full((len(lens), maxp), -1, dtype=np.int32)
        there = np.zeros((P, page), dtype=bool)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = order[at:at + u]
            for j in range(u):
                there[order[at + j], : min(page, lens[b] - j * page)] = True
            at += u
        self.host, self.pages, self.dev = [], [], []
        for i, nb in enumerate(bits):
            rows = rows_of((P, hkv, page, d), 10 * tag + i) if special else oracle.to_bf16_bits(g.normal(0, sigma, (P, hkv, page, d)))
            codes, scales = kv_mx.quantise(rows, nb)
            values = oracle.to_bf16_bits(kv_mx.values(codes, scales, nb))
            gone = np.broadcast_to(~there[:, None], rows.shape[:3])
            codes[gone], scales[gone], values[gone] = 0xFF, 0xFF, 0x7FC0
            self.host += [codes, scales]
            self.pages.append(values)
        self.dev = tuple(dev_u8(c) for c in self.host)
        self.kp, self.vp = (gu.dev(v) for v in self.pages)
        self.q = g


def both(ua, c, q, lens, most, table=None, scale=None):
    """The decode over the codes and the bf16 decode over the values, outputs and lse as bits."""
    import torch
    table = gu.dev_i32(c.table) if table is None else table
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    need = ua.decode_mx_workspace_bytes(q.shape[0], most, q.shape[1], c.host[0].shape[1], q.shape[2])
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")    # any contents: NaN partials
    ua.decode_mx(q, *c.dev, table, lens, most, softmax_scale=scale, out=out, lse=lse, workspace=ws)
    want, wlse = ua.decode(q, c.kp, c.vp, table, lens, most, softmax_scale=scale, return_lse=True)
    return (gu.host_bits(out), lse.cpu().numpy().view(np.uint32)), (gu.host_bits(want), wlse.cpu().numpy().view(np.uint32))


CASES = [  # lengths, q heads, kv heads, d, page
    ([1], 1, 1, 128, 16), ([1, 2, 15, 16, 17], 4, 1, 64, 16), ([63, 64, 65, 255, 256, 257], 8, 2, 128, 16),
    ([300, 1, 511, 512, 513], 16, 1, 128, 64), ([700], 32, 8, 128, 256), ([33, 1025, 90], 17, 1, 64, 32),
    ([2000, 7, 449], 64, 2, 128, 16), ([1300, 1301], 6, 3, 64, 64), ([4100], 2, 1, 128, 64), ([260, 100], 34, 2, 128, 128),
]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_decode_has_the_bf16_decodes_bits(ua, bits, case):
    lens, hq, hkv, d, page = CASES[case]
    c = Cache(lens, hkv, d, page, bits, 20 + case)
    q = gu.dev(inputs.normal_bf16((len(lens), hq, d), 1.0, 620, case))
    for most in (max(lens), max(lens) + page, (max(lens) // page + 2) * page):
        got, want = both(ua, c, q, gu.dev_i32(lens), most)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    assert not np.any(np.isnan(oracle.bf16_to_f64(got[0])))


@pytest.mark.parametrize("bits", BITS)
def test_decode_against_the_oracle(ua, bits):
    """The fp64 attention over the oracle's own values, within the bf16 decode's gate."""
    lens, hq, hkv, d, page = [1, 77, 300, 1111], 12, 3, 128, 32
    c = Cache(lens, hkv, d, page, bits, 31)
    q_bits = inputs.normal_bf16((4, hq, d), 1.0, 621)
    out, lse = ua.decode_mx(gu.dev(q_bits), *c.dev, gu.dev_i32(c.table), gu.dev_i32(lens), max(lens), return_lse=True)
    want, wlse = oracle.paged_decode_fp64(q_bits, c.pages[0], c.pages[1], c.table, np.array(lens))
    rep = oracle.parity_report(gu.host_f64(out), want)
    assert rep["pass"], rep
    assert np.max(np.abs(lse.cpu().numpy() - wlse)) <= oracle.LSE_ABS


def test_decode_rising_scores_and_other_scales(ua):
    """References that move in every tile, a scale that makes one key take all, and one that makes all keys equal."""
    lens = [1500, 600]
    for bits in ((8, 8), (4, 4)):
        c = Cache(lens, 2, 128, 64, bits, 33, sigma=4.0)
        q = gu.dev(inputs.normal_bf16((2, 8, 128), 4.0, 622))
        for scale in (1e-4, 0.09, 1.0, 30.0):
            got, want = both(ua, c, q, gu.dev_i32(lens), 1500, scale=scale)
            assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def _many(ua, lens, hq, hkv, d, bits, tag, most=None, sigma=4.0):
    """Both decodes of sequences given by their lengths (0: none) where all share one long sequence's pages."""
    long = max(lens)
    c = Cache([long], hkv, d, 16, bits, tag, sigma=sigma)
    table = gu.dev_i32(np.repeat(c.table, len(lens), axis=0))
    q = gu.dev(inputs.normal_bf16((len(lens), hq, d), sigma, 628, tag))
    got, want = both(ua, c, q, gu.dev_i32(lens), most or long, table=table, scale=0.05)
    there = np.array(lens) > 0
    assert np.array_equal(got[0][there], want[0][there]) and np.array_equal(got[1][there], want[1][there])
    assert np.all(np.isnan(oracle.bf16_to_f64(got[0][~there])))
    assert not np.any(np.isnan(oracle.bf16_to_f64(got[0][there])))


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("hq,hkv,d", [(16, 8, 128), (16, 16, 64), (136, 8, 64), (136, 8, 128)])
def test_decode_many_long_sequences(ua, bits, hq, hkv, d):
    """More pairs of sequence and kv head than workgroups fit the chip, past eight chunks: lengths around the borders of tiles,
    chunks and of four chunks, references that move, entries without keys."""
    n = 1100 // hkv
    lens = [2100, 1, 0, 64, 65, 1023, 1024, 1025, 257, 2049, 2048, -3, 2304] + list(inputs.rng(640, d).integers(1, 600, n - 13))
    _many(ua, lens, hq, hkv, d, bits, 60 + hkv)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("hq,d", [(4, 128), (34, 128), (8, 64), (40, 64)])
def test_decode_more_chunks_than_waves(ua, bits, hq, d):
    """Six hundred pairs of sequence and kv head, 67 chunks: some sequences have more chunks than a pair has waves."""
    lens = [17000, 1, 0, 54 * 256, 54 * 256 + 1, 55 * 256, 15000, 256, 257, -3] + list(inputs.rng(641, d).integers(1, 900, 290))
    _many(ua, lens, hq, 2, d, bits, 90)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("hq,hkv,d,long", [(4, 2, 128, 2048), (34, 2, 64, 1500), (34, 2, 128, 1500), (16, 1, 64, 300), (8, 1, 128, 900)])
def test_decode_few_chunks(ua, bits, hq, hkv, d, long):
    """Up to eight chunks, entries of fewer among them."""
    _many(ua, [long, 1, 0, 256, 257, long - 1, 64, min(long, 512), 280], hq, hkv, d, bits, 70 + hkv)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (17, 1, 128), (5, 1, 64), (32, 1, 64)])
def test_decode_bound_far_above_the_lengths(ua, bits, hq, hkv, d):
    """max_seqlen of a million (codes are then read past the caches), lengths of up to eleven chunks."""
    lens = [2700, 1, 256, 257, 513, 0, 1100]
    c = Cache([max(lens)], hkv, d, 16, bits, 80, sigma=4.0)
    table = np.full((len(lens), 1 << 16), -1, dtype=np.int32)
    table[:, : c.table.shape[1]] = c.table
    q = gu.dev(inputs.normal_bf16((len(lens), hq, d), 4.0, 629, hq))
    got, want = both(ua, c, q, gu.dev_i32(lens), 1 << 20, table=gu.dev_i32(table), scale=0.05)
    there = np.array(lens) > 0
    assert np.array_equal(got[0][there], want[0][there]) and np.array_equal(got[1][there], want[1][there])


def test_decode_nan_blocks_reach_their_rows_alone(ua):
    """Blocks that read as NaN inside a context: NaN for the kv head they are in, as in the bf16 decode; others untouched."""
    lens = [300, 40]
    for bits in BITS:
        c = Cache(lens, 2, 64, 16, bits, 34)
        q = gu.dev(inputs.normal_bf16((2, 4, 64), 1.0, 623))
        page = int(c.table[0, 260 // 16])
        c.dev[3][page, 1, 260 % 16, 1] = 255                  # of V: kv head 1, d 32 .. 63
        c.vp[page, 1, 260 % 16, 32:] = float("nan")
        got, want = both(ua, c, q, gu.dev_i32(lens), 300)
        assert same_values(got[0], want[0])
        v = oracle.bf16_to_f64(got[0])
        assert np.all(np.isnan(v[0, 2:, 32:])) and not np.any(np.isnan(v[0, :2])) and not np.any(np.isnan(v[1]))
        assert not np.any(np.isnan(v[0, 2:, :32]))
        c.dev[1][page, 1, 260 % 16, 0] = 255                  # of K: all of the head's scores with that key
        c.kp[page, 1, 260 % 16, :32] = float("nan")
        got, want = both(ua, c, q, gu.dev_i32(lens), 300)
        assert same_values(got[0], want[0]) and np.all(np.isnan(oracle.bf16_to_f64(got[0])[0, 2:]))


def test_decode_special_values(ua):
    """Large and tiny numbers, zeros and blocks without numbers anywhere in the cache."""
    lens = [700, 130]
    for bits in BITS:
        c = Cache(lens, 2, 128, 32, bits, 35, special=True)
        q = gu.dev(inputs.normal_bf16((2, 6, 128), 1.0, 624))
        got, want = both(ua, c, q, gu.dev_i32(lens), 700)
        assert same_values(got[0], want[0])


def test_decode_tables_with_bad_pages(ua):
    """Pages outside the pool inside a context read as zeros, entries behind it are not read."""
    lens = [500, 70]
    for bits in ((8, 8), (4, 4)):
        c = Cache(lens, 2, 128, 16, bits, 36)
        table = c.table.copy()
        table[0, 3], table[0, 20], table[1, 2] = -1, 10 ** 9, -(2 ** 31)
        q = gu.dev(inputs.normal_bf16((2, 8, 128), 1.0, 625))
        got, want = both(ua, c, q, gu.dev_i32(lens), 500, table=gu.dev_i32(table))
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
        assert not np.any(np.isnan(oracle.bf16_to_f64(got[0])))


def test_decode_lengths_out_of_range(ua):
    """Longer than max_seqlen: clamped to it; none or negative: the row is left as it was."""
    lens = [600, 300, 50, 90]
    c = Cache(lens, 1, 64, 16, (8, 4), 37)
    q = gu.dev(inputs.normal_bf16((4, 3, 64), 1.0, 626))
    got, want = both(ua, c, q, gu.dev_i32([600, 0, -5, 90]), 400)
    clamped, _ = both(ua, c, q, gu.dev_i32([400, 300, 50, 90]), 400)
    for i in (0, 3):
        assert np.array_equal(got[0][i], want[0][i]) and np.array_equal(got[1][i], want[1][i])
        assert np.array_equal(got[0][i], clamped[0][i])
    assert np.all(np.isnan(oracle.bf16_to_f64(got[0][1:3]))) and np.all(np.isnan(got[1][1:3].view(np.float32)))


def test_decode_does_not_depend_on_the_batch(ua):
    lens = [900, 17, 256, 1400, 64]
    c = Cache(lens, 2, 128, 64, (4, 4), 38)
    q = gu.dev(inputs.normal_bf16((5, 16, 128), 1.0, 627))
    table = gu.dev_i32(c.table)
    all_ = gu.host_bits(ua.decode_mx(q, *c.dev, table, gu.dev_i32(lens), 1400))
    for order in ([4, 2, 0, 3, 1], [3], [1, 4]):
        i = np.array(order)
        part = ua.decode_mx(q[i].contiguous(), *c.dev, table[i].contiguous(), gu.dev_i32(np.array(lens)[i]), 1500)
        assert np.array_equal(gu.host_bits(part), all_[i])


@pytest.mark.parametrize("bits,d,hq,hkv", [((8, 8), 128, 8, 2), ((4, 4), 64, 4, 2), ((8, 4), 128, 34, 2)])
def test_rollout_and_update_agree(ua, bits, d, hq, hkv):
    """Prompts written, each response token written and decoded; the update rounds its rows and runs the full sequence: the same
    bits in every decoded row.  The cache read back is the rounded rows."""
    import torch
    w = inputs.custom(hq, hkv, d, [64 + 30, 150 + 41, 33 + 20, 270 + 9], sigma=1.0, page_size=16, prompt_lens=[64, 150, 33, 270])
    pk = gu.Pack(w, seed=13)
    kr, vr = ua.kv_round_mx(pk.k, pk.v, *bits)
    full, flse = ua.prefill(pk.q, kr, vr, pk.cu_dev, pk.max_seqlen, return_lse=True)
    full, flse = gu.host_bits(full), flse.cpu().numpy().view(np.uint32)
    cache = ua.mx_cache(pk.kp.shape[0], hkv, 16, d, *bits)
    for t in cache:
        t.fill_(0xFF)
    P, table = w.prompt_lens, pk.table_dev
    seq = np.concatenate([np.full(P[b], b) for b in range(w.num_seqs)]).astype(np.int32)
    pos = np.concatenate([np.arange(P[b]) for b in range(w.num_seqs)]).astype(np.int32)
    it = torch.from_numpy(pk.cu[seq] + pos).cuda()
    ua.kv_write_mx(pk.k[it], pk.v[it], table, gu.dev_i32(seq), gu.dev_i32(pos), *cache)
    R = [L - p for L, p in zip(w.seq_lens, P)]
    for step in range(max(R)):
        sq = np.array([b for b in range(w.num_seqs) if step < R[b]], dtype=np.int32)
        ps = np.array([P[b] + step for b in sq], dtype=np.int32)
        tk = torch.from_numpy(pk.cu[sq] + ps).cuda()
        ua.kv_write_mx(pk.k[tk], pk.v[tk], table, gu.dev_i32(sq), gu.dev_i32(ps), *cache)
        out, lse = ua.decode_mx(pk.q[tk].contiguous(), *cache, table[torch.from_numpy(sq.astype(np.int64)).cuda()].contiguous(),
                                gu.dev_i32(ps + 1), max(w.seq_lens), return_lse=True)
        assert np.array_equal(gu.host_bits(out), full[pk.cu[sq] + ps])
        assert np.array_equal(lse.cpu().numpy().view(np.uint32), flse[pk.cu[sq] + ps])
    seq = np.concatenate([np.full(L, b) for b, L in enumerate(w.seq_lens)])
    pos = np.concatenate([np.arange(L) for L in w.seq_lens])
    k, v = ua.kv_read_mx(*cache, table, gu.dev_i32(seq), gu.dev_i32(pos))
    assert np.array_equal(gu.host_bits(k), gu.host_bits(kr)) and np.array_equal(gu.host_bits(v), gu.host_bits(vr))
    assert np.array_equal(gu.host_bits(kr), oracle.mx_round(pk.host["k"], bits[0]))


def test_gradient_through_the_rounding(ua):
    """The backward over the rounded rows is the gradient of the attention at them (the formula's, in fp64)."""
    w = inputs.custom(4, 2, 64, [70, 130, 1], sigma=1.0, page_size=16)
    pk = gu.Pack(w, seed=14)
    kr, vr = ua.kv_round_mx(pk.k, pk.v, 8, 4)
    out, lse = ua.prefill(pk.q, kr, vr, pk.cu_dev, 130, return_lse=True)
    dout = inputs.normal_bf16(tuple(pk.q.shape), 1.0, 631)
    grads = ua.prefill_backward(pk.q, kr, vr, out, gu.dev(dout), lse, pk.cu_dev, 130)
    at = pk.host["q"], oracle.mx_round(pk.host["k"], 8), oracle.mx_round(pk.host["v"], 4), dout, pk.cu
    for got, want, size in zip(grads, oracle.attention_backward_fp64(*at), oracle.backward_error_scales(*at)):
        assert np.all(np.abs(gu.host_f64(got) - want) <= 2.0 ** -7 * size + 2.0 ** -8 * np.abs(want) + 1e-300)


def test_workspace_shared_with_the_bf16_decode(ua):
    """One workspace in turn for both decodes: the counters that the bf16 decode keeps there survive."""
    lens = [1000, 600, 2000]
    c = Cache(lens, 2, 128, 64, (4, 4), 40)
    q = gu.dev(inputs.normal_bf16((3, 8, 128), 1.0, 632))
    table, n = gu.dev_i32(c.table), gu.dev_i32(lens)
    ws = ua.new_workspace(ua.decode_workspace_bytes(3, 2000, 8, 128))
    want = gu.host_bits(ua.decode(q, c.kp, c.vp, table, n, 2000))
    for _ in range(3):
        assert np.array_equal(gu.host_bits(ua.decode_mx(q, *c.dev, table, n, 2000, workspace=ws)), want)
        assert np.array_equal(gu.host_bits(ua.decode(q, c.kp, c.vp, table, n, 2000, workspace=ws)), want)


def test_graph_of_a_step(ua):
    """A step (write, decode) captured once and replayed with new rows, places and lengths, eager work between the replays."""
    import torch
    lens = [700, 90, 1500]
    B, hkv, hq, d, page = 3, 2, 8, 128, 16
    c = Cache([n + 8 for n in lens], hkv, d, page, (8, 4), 41)
    table = gu.dev_i32(c.table)
    q = torch.zeros((B, hq, d), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((B, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seq, pos, n = gu.dev_i32(range(B)), gu.dev_i32([0] * B), gu.dev_i32([1] * B)
    mine, other = tuple(t.clone() for t in c.dev), tuple(t.clone() for t in c.dev)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            ua.kv_write_mx(k, v, table, seq, pos, *mine)
            out = ua.decode_mx(q, *mine, table, n, 1520)
            back = ua.kv_read_mx(*mine, table, seq, pos)
            rounded = ua.kv_round_mx(k, v, 8, 4)
    torch.cuda.synchronize()
    for rep in range(4):
        fresh = [gu.dev(inputs.normal_bf16(tuple(t.shape), 1.0, 633, rep, i)) for i, t in enumerate((q, k, v))]
        at = np.array(lens) - 300 * (rep == 2) * (np.array(lens) > 400) + rep
        for t, x in zip((q, k, v), fresh):
            t.copy_(x)
        pos.copy_(gu.dev_i32(at))
        n.copy_(gu.dev_i32(at + 1))
        graph.replay()
        torch.cuda.synchronize()
        ua.kv_write_mx(fresh[1], fresh[2], table, seq, gu.dev_i32(at), *other)
        want = ua.decode_mx(fresh[0], *other, table, gu.dev_i32(at + 1), 1520)
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        for a, b in zip(mine, other):
            assert torch.equal(a, b)
        for a, b in zip(back, rounded):
            assert torch.equal(a, b)


def test_streams(ua):
    """A call for another stream than the current one: ordered there, its outputs made there."""
    import torch
    c = Cache([600, 80], 2, 64, 16, (8, 8), 42)
    q = gu.dev(inputs.normal_bf16((2, 4, 64), 1.0, 634))
    table, n = gu.dev_i32(c.table), gu.dev_i32([600, 80])
    want = ua.decode_mx(q, *c.dev, table, n, 600)
    k = gu.dev(inputs.normal_bf16((2, 2, 64), 1.0, 635))
    seq, pos = gu.dev_i32([0, 1]), gu.dev_i32([3, 4])
    rounded = ua.kv_round_mx(k, k.clone(), 8, 8)
    side, a = torch.cuda.Stream(), torch.ones((4096, 4096), device="cuda")
    late_q, late_k, late = torch.zeros_like(q), torch.zeros_like(k), tuple(torch.zeros_like(t) for t in c.dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):          # some milliseconds of that stream's time, then the inputs
            a = a @ a * 2.0 ** -12
        late_q.copy_(q)
        late_k.copy_(k)
        for t, x in zip(late, c.dev):
            t.copy_(x)
    got = ua.decode_mx(late_q, *late, table, n, 600, stream=side)
    ua.kv_write_mx(late_k, late_k, table, seq, pos, *late, stream=side)
    back = ua.kv_read_mx(*late, table, seq, pos, stream=side)
    r = ua.kv_round_mx(late_k, late_k, 8, 8, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(back[0], rounded[0]) and torch.equal(back[1], rounded[0])
    assert torch.equal(r[0], rounded[0])


def test_validation(ua, monkeypatch):
    """UATTN_VALIDATE refuses places and lengths that the calls would skip or clamp."""
    import torch
    cache = ua.mx_cache(4, 1, 16, 64, 8, 4)
    k = torch.ones((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    table, seq = gu.dev_i32([[0, 1], [2, 3], [0, 7]]), gu.dev_i32([0, 1, 2])
    q, good = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda"), gu.dev_i32([0, 17, -1])
    calls = [lambda s, p: ua.kv_write_mx(k, k, table, s, p, *cache), lambda s, p: ua.kv_read_mx(*cache, table, s, p)]
    bad = [(seq, gu.dev_i32([0, 32, 0])), (seq, gu.dev_i32([0, 0, 16])), (gu.dev_i32([0, 1, 3]), gu.dev_i32([0, 0, 0]))]
    for call in calls:
        for s, p in bad:
            call(s, p)
    monkeypatch.setenv("UATTN_VALIDATE", "1")
    for call in calls:
        call(seq, good)
        for s, p in bad:
            with pytest.raises(ua.UattnError, match="EINVAL"):
                call(s, p)
    ua.decode_mx(q, *cache, table, gu.dev_i32([1, 32, 16]), 32)
    for lens in ([1, 33, 16], [0, 1, 1], [1, 32, 17]):
        with pytest.raises(ua.UattnError, match="EINVAL"):
            ua.decode_mx(q, *cache, table, gu.dev_i32(lens), 32)


def test_refusals(ua):
    import torch
    cache = ua.mx_cache(4, 2, 16, 64, 8, 4)
    rows = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    table, seq, pos = gu.dev_i32([[0, 1]] * 3), gu.dev_i32([0, 1, 2]), gu.dev_i32([0, 1, 2])
    q = torch.ones((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    lens = gu.dev_i32([1, 1, 1])
    kc, ks, vc, vs = cache
    wrong = [
        lambda: ua.kv_write_mx(rows.float(), rows, table, seq, pos, *cache),
        lambda: ua.kv_write_mx(rows.transpose(1, 2), rows.transpose(1, 2), table, seq, pos, *cache),
        lambda: ua.kv_write_mx(rows, torch.ones((3, 4, 64), dtype=torch.bfloat16, device="cuda")[:, :2], table, seq, pos, *cache),
        lambda: ua.kv_write_mx(rows[:, :1], rows[:, :1], table, seq, pos, *cache),
        lambda: ua.kv_write_mx(rows, rows, table, seq.long(), pos, *cache),
        lambda: ua.kv_write_mx(rows, rows, table, seq[:2], pos, *cache),
        lambda: ua.kv_write_mx(rows, rows, table, seq, pos, kc[..., :48], ks, vc, vs),
        lambda: ua.kv_write_mx(rows, rows, table, seq, pos, kc, ks[:3], vc, vs),
        lambda: ua.kv_write_mx(rows, rows, table, seq, pos, kc.view(torch.int8), ks, vc, vs),
        lambda: ua.kv_write_mx(rows, rows, table, seq, pos, kc[:, :, ::2], ks[:, :, ::2], vc[:, :, ::2], vs[:, :, ::2]),
        lambda: ua.kv_write_mx(rows, rows, table, seq, pos, kc.cpu(), ks, vc, vs),
        lambda: ua.kv_read_mx(*cache, table, seq, pos[:, None]),
        lambda: ua.kv_read_mx(*cache, table, seq, pos, k_out=rows[:2], v_out=rows[:2]),
        lambda: ua.kv_round_mx(rows, rows.clone(), 8, 16),
        lambda: ua.kv_round_mx(rows.cpu(), rows.cpu()),
        lambda: ua.decode_mx(q[..., :32].contiguous(), *cache, table, lens, 1),
        lambda: ua.decode_mx(q, *cache, table[:2], lens, 1),
        lambda: ua.decode_mx(q, *cache, table, lens.long(), 1),
        lambda: ua.decode_mx(q, *cache, table, lens, 1, out=q[:2]),
        lambda: ua.decode_mx(q, *cache, table, lens, 1, lse=torch.empty((3, 4), device="cuda", dtype=torch.float64)),
        lambda: ua.mx_cache(4, 2, 16, 64, 8, 2), lambda: ua.mx_cache(4, 2, 16, 96),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ua.kv_round_mx(rows, rows, 8, 8, k_out=rows, v_out=rows),     # both outputs one tensor
                 lambda: ua.decode_mx(q, *cache, table, lens, 33),                     # the table is shorter
                 lambda: ua.decode_mx(q[:, :3].contiguous(), *cache, table, lens, 1),
                 lambda: ua.decode_mx(q, *ua.mx_cache(4, 2, 24, 64), table, lens, 1)):
        with pytest.raises(ua.UattnError):
            call()
