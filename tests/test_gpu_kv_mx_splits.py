"""The decode over a cache in 8 or 4 bits in each of the ways that its launch splits the work: workspaces shared with the bf16
decode, captured steps, other streams, blocks that read as NaN, long contexts.  A way is held to what tells it from outside:
whether sizes need a workspace, and whether the call writes to it."""
import math

import numpy as np
import pytest

from paper_2609_35140_amd import inputs

pytestmark = pytest.mark.gpu
gu = pytest.importorskip("gpu_util")
from test_gpu_kv_mx import Cache, both, same_values, ua  # noqa: E402,F401

# (entries, q heads, kv heads, d, longest, bound); whether partials go through the workspace
SPLITS = {
    "fold": ((3, 8, 2, 128, 1500, 1520), False),           # a workgroup folds up to eight chunks in LDS
    "fold_wide": ((3, 34, 2, 64, 1500, 1520), False),
    "chunks": ((3, 8, 2, 128, 2900, 3000), True),          # a wave to a chunk, and the merge
    "chunks_wide": ((3, 34, 2, 128, 2900, 3000), True),
    "walk": ((3, 8, 2, 64, 2900, 1 << 21), True),          # a wave takes several chunks: more than 32768 under the bound
    "walk_wide": ((3, 34, 2, 128, 2900, 1 << 21), True),
    "turns": ((520, 8, 2, 128, 2900, 3000), False),        # four pairs to a CU: a workgroup to a pair, state in LDS
    "turns_wide": ((520, 34, 2, 64, 2900, 3000), False),
}
BITS = [(8, 4), (4, 4)]


def _lens(name, tag=0):
    """Lengths: the longest, one near it, borders of tiles and chunks, none."""
    (B, _, _, _, long, _), _ = SPLITS[name]
    lens = [long, 90, long - 250]
    if B > 3:
        lens += [1, 64, 65, 255, 256, 257, 1023, 1024, 1025, 0, 2560, 2561]
        lens += list(inputs.rng(650, tag).integers(1, 600, B - len(lens)))
    return lens


class Setup:
    """One long sequence that all entries read, in codes and as values."""

    def __init__(self, ua, name, bits, tag, special=False):
        (self.B, self.hq, self.hkv, self.d, self.long, self.most), self.stores = SPLITS[name]
        self.c = Cache([self.long], self.hkv, self.d, 16, bits, tag, slack=0, special=special)
        self.lens = np.array(_lens(name, tag))
        table = np.full((self.B, -(-self.most // 16)), -1, dtype=np.int32)
        table[:, : self.c.table.shape[1]] = self.c.table
        self.table = gu.dev_i32(table)
        self.q = gu.dev(inputs.normal_bf16((self.B, self.hq, self.d), 1.0, 651, tag))
        self.need = ua.decode_mx_workspace_bytes(self.B, self.most, self.hq, self.hkv, self.d)
        self.turns = name.startswith("turns")
        assert (self.need > 0) == (self.stores or self.turns)

    def mx(self, ua, lens=None, **kw):
        return ua.decode_mx(self.q, *self.c.dev, self.table, gu.dev_i32(self.lens if lens is None else lens), self.most, **kw)

    def bf16(self, ua, lens=None, **kw):
        return ua.decode(self.q, self.c.kp, self.c.vp, self.table, gu.dev_i32(self.lens if lens is None else lens), self.most, **kw)

    def bits(self, out):
        return gu.host_bits(out)[self.lens > 0]


@pytest.mark.parametrize("name", SPLITS)
def test_which_split(ua, name):
    """Partials are stored by the ways that merge them in a second launch, and by no other."""
    import torch
    s = Setup(ua, name, (4, 4), 100)
    ws = torch.full((max(s.need, 4096),), 0xFF, dtype=torch.uint8, device="cuda")
    s.mx(ua, workspace=ws)
    assert bool((ws != 0xFF).any()) == s.stores


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("name", SPLITS)
def test_workspace_of_both_decodes(ua, name, bits):
    """In turn on one workspace: of the bf16 decode's size, of the mx decode's own, and of odd sizes between."""
    s = Setup(ua, name, bits, 101)
    want = s.bits(s.bf16(ua))
    small = s.lens[:1] // 3
    args = s.q[:1].contiguous(), s.c.kp, s.c.vp, s.table[:1].contiguous(), gu.dev_i32(small), 1000
    want_small = gu.host_bits(ua.decode(*args))
    both_need = ua.decode_workspace_bytes(s.B, s.most, s.hq, s.d)
    least = max(s.need, ua.decode_workspace_bytes(1, 1000, s.hq, s.d))
    for size in (both_need, least, least + 48, both_need + 4096):
        ws = ua.new_workspace(size)
        for _ in range(2):
            assert np.array_equal(s.bits(s.mx(ua, workspace=ws)), want)
            assert np.array_equal(gu.host_bits(ua.decode(*args, workspace=ws)), want_small)
            assert np.array_equal(s.bits(s.mx(ua, workspace=ws)), want)
            if size >= both_need:
                assert np.array_equal(s.bits(s.bf16(ua, workspace=ws)), want)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("name", SPLITS)
def test_captured_step(ua, name, bits):
    """The write of a token and the decode over it, replayed with new rows and lengths, eager work between the replays."""
    import torch
    s = Setup(ua, name, bits, 102)
    k, v = (torch.zeros((s.B, s.hkv, s.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seq, pos = gu.dev_i32(range(s.B)), gu.dev_i32([-1] * s.B)       # one entry's token is written, the others' are padding
    q, n = torch.zeros_like(s.q), gu.dev_i32([1] * s.B)
    mine, other = tuple(t.clone() for t in s.c.dev), tuple(t.clone() for t in s.c.dev)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ua.kv_write_mx(k, v, s.table, seq, pos, *mine)
        out, lse = ua.decode_mx(q, *mine, s.table, n, s.most, return_lse=True)
    torch.cuda.synchronize()
    for rep in range(4):
        fresh = [gu.dev(inputs.normal_bf16(tuple(t.shape), 1.0, 652, rep, i)) for i, t in enumerate((q, k, v))]
        lens = np.maximum(np.roll(s.lens, rep), 1) if rep % 2 else np.maximum(s.lens - 40 * rep, 1)
        at = [int(lens.max()) - 1 if b == int(lens.argmax()) else -1 for b in range(s.B)]
        for t, x in zip((q, k, v), fresh):
            t.copy_(x)
        pos.copy_(gu.dev_i32(at))
        n.copy_(gu.dev_i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        ua.kv_write_mx(fresh[1], fresh[2], s.table, seq, gu.dev_i32(at), *other)
        want, wlse = ua.decode_mx(fresh[0], *other, s.table, gu.dev_i32(lens), s.most, return_lse=True)
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse.view(torch.int32), wlse.view(torch.int32))
        assert not bool(torch.isnan(out).any())
        for a, b in zip(mine, other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", SPLITS)
def test_on_another_stream(ua, name):
    """Ordered behind the inputs that another stream makes, all its launches there; twice, one behind the other."""
    import torch
    s = Setup(ua, name, (8, 4), 103)
    want = s.bits(s.mx(ua))
    side, a = torch.cuda.Stream(), torch.ones((4096, 4096), device="cuda")
    n, late_q, late = gu.dev_i32(s.lens), torch.zeros_like(s.q), tuple(torch.zeros_like(t) for t in s.c.dev)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):          # some milliseconds of that stream's time, then the inputs
            a = a @ a * 2.0 ** -12
        late_q.copy_(s.q)
        for t, x in zip(late, s.c.dev):
            t.copy_(x)
    first = ua.decode_mx(late_q, *late, s.table, n, s.most, stream=side)
    second = ua.decode_mx(late_q, *late, s.table, n, s.most, stream=side)
    torch.cuda.synchronize()
    assert np.array_equal(s.bits(first), want) and np.array_equal(s.bits(second), want)


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("name", SPLITS)
def test_blocks_without_numbers(ua, name, bits):
    """Of K at a late position and of V at an early one, both of kv head 1: NaN in the rows that attend to them and no others."""
    s = Setup(ua, name, bits, 104)
    c, d, G = s.c, s.d, s.hq // s.hkv
    late, early = s.long - 100, 70
    for at, part, block in ((late, 1, 0), (early, 3, 1)):
        page = int(c.table[0, at // 16])
        c.dev[part][page, 1, at % 16, block] = 255
        (c.kp if part == 1 else c.vp)[page, 1, at % 16, 32 * block: 32 * block + 32] = float("nan")
    (got, lse), (want, wlse) = both(ua, c, s.q, gu.dev_i32(s.lens), s.most, table=s.table)
    there = s.lens > 0
    assert same_values(got[there], want[there])
    nan = np.isnan(gu.host_f64(gu.dev(got)))
    assert np.all(nan[s.lens > late, G:]) and not np.any(nan[there][:, :G])
    mid = (s.lens > early) & (s.lens <= late)
    assert np.all(nan[mid][:, G:, 32:64]) and not np.any(nan[mid][:, :, :32]) and not np.any(nan[mid][:, :, 64:])
    few = there & (s.lens <= early)
    assert not np.any(nan[few])
    lse, wlse = lse.view(np.float32)[there], wlse.view(np.float32)[there]
    assert np.array_equal(lse, wlse, equal_nan=True)
    assert np.array_equal(np.isnan(lse[:, G:]), np.broadcast_to((s.lens[there] > late)[:, None], lse[:, G:].shape))


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("name", SPLITS)
def test_any_values(ua, name, bits):
    """Everything that a block may hold, anywhere in the cache."""
    s = Setup(ua, name, bits, 105, special=True)
    (got, _), (want, _) = both(ua, s.c, s.q, gu.dev_i32(s.lens), s.most, table=s.table)
    assert same_values(got[s.lens > 0], want[s.lens > 0])


def _long_cache(ua, n, hkv, d, bits, tag):
    """A sequence of n keys on pages in any order, in codes and as bf16 pages, and its rows; made on the GPU."""
    import torch
    page = 64
    maxp = -(-n // page)
    g = torch.Generator(device="cuda")
    g.manual_seed(tag)
    table = torch.randperm(maxp, generator=g, device="cuda").to(torch.int32)[None]
    rows = [torch.randn((maxp * page, hkv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    cache = ua.mx_cache(maxp, hkv, page, d, *bits)
    pos = torch.arange(maxp * page, dtype=torch.int32, device="cuda")
    seq = torch.zeros_like(pos)
    ua.kv_write_mx(*rows, table, seq, pos, *cache)
    rows = ua.kv_read_mx(*cache, table, seq, pos)
    pages = []
    for r in rows:
        p = torch.empty((maxp, hkv, page, d), dtype=torch.bfloat16, device="cuda")
        p[table[0].long()] = r.view(maxp, page, hkv, d).transpose(1, 2)
        pages.append(p)
    return cache, pages, rows, table


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("B,hq,hkv,d,bound", [(9, 8, 2, 128, 300001), (9, 17, 1, 128, 300001), (9, 5, 1, 64, 300001),
                                              (40, 8, 2, 64, 1 << 20), (40, 20, 1, 128, 1 << 20),
                                              (520, 4, 2, 128, 70001), (520, 34, 2, 64, 70001)])
def test_long_contexts(ua, bits, B, hq, hkv, d, bound):
    """Past 32,768 keys: more groups of 64 chunks than two, their borders; under a bound of a million up to 1172 chunks to the 409
    or 819 waves of a pair.  Three of the rows against 64 bits."""
    import torch
    cache, pages, rows, table = _long_cache(ua, min(bound, 300001), hkv, d, bits, 110)
    lens = [32768, 32769, 33024, 33025, 49152, 49153, 65536 + 256, min(bound, 300001), 70001]
    lens += list(inputs.rng(653).integers(1, 700, B - 9))
    q = gu.dev(inputs.normal_bf16((B, hq, d), 1.0, 654))
    full = torch.full((B, -(-bound // 64)), -1, dtype=torch.int32, device="cuda")
    full[:, : table.shape[1]] = table
    n = gu.dev_i32(lens)
    out, lse = ua.decode_mx(q, *cache, full, n, bound, return_lse=True)
    want, wlse = ua.decode(q, *pages, full, n, bound, return_lse=True)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse.view(torch.int32), wlse.view(torch.int32))
    # 64 bits: weights rounded to bf16 (2^-8 each, in the sum over V and in the normaliser alike), the row rounded once
    # (2^-8); scores of d products and the sums over chunks in fp32, far below 2^-12
    for b in (2, 5, 7):
        k, v = (r[: lens[b]].transpose(0, 1).double().repeat_interleave(hq // hkv, 0) for r in rows)
        w = torch.softmax(torch.matmul(k, q[b].double()[:, :, None])[..., 0] / math.sqrt(d), 1)[:, None]
        ref, size = torch.matmul(w, v)[:, 0], torch.matmul(w, v.abs())[:, 0]
        err = (out[b].double() - ref).abs()
        assert bool((err <= (2.0 ** -8 * (size + 2 * ref.abs())) * (1 + 2.0 ** -6) + 2.0 ** -12 * size).all())
        x = torch.logsumexp(torch.matmul(k, q[b].double()[:, :, None])[..., 0] / math.sqrt(d), 1)
        assert bool(((lse[b].double() - x).abs() <= 2.0 ** -8 * (1 + 2.0 ** -6) + 2.0 ** -16 * x.abs()).all())


@pytest.mark.parametrize("which", [0, 1])
def test_one_output_given(ua, which):
    """The rows read back and rounded, one output inside the projection's rows, the other made beside it."""
    import torch
    g = inputs.rng(655)
    N, hkv, d = 40, 2, 64
    k, v = (gu.dev(inputs.normal_bf16((N, hkv, d), 1.0, 656, i)) for i in range(2))
    cache = ua.mx_cache(6, hkv, 16, d, 8, 4)
    places = gu.dev_i32(g.permutation(6)[:3].reshape(1, 3)), gu.dev_i32([0] * N), gu.dev_i32(g.permutation(48)[:N])
    ua.kv_write_mx(k, v, *places, *cache)
    want = ua.kv_round_mx(k, v, 8, 4)
    for call in (lambda **o: ua.kv_read_mx(*cache, *places, **o), lambda **o: ua.kv_round_mx(k, v, 8, 4, **o)):
        fused = torch.full((N, 8, d), 3.0, dtype=torch.bfloat16, device="cuda")
        got = call(**{("k_out", "v_out")[which]: fused[:, 3:5]})
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(fused[:, 3:5], want[which])
        assert bool((fused[:, :3] == 3.0).all()) and bool((fused[:, 5:] == 3.0).all())
