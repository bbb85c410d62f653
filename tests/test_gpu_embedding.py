"""GPU embedding lookup and its table's gradient against the float64 oracle."""
import numpy as np
import pytest

import oracle
from paper_2609_35140_amd import inputs

pytestmark = pytest.mark.gpu
gu = pytest.importorskip("gpu_util")

U = 2.0 ** -24
HALF = 2.0 ** -8


@pytest.fixture(scope="module")
def ua():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35140_amd import uattn
    uattn.lib()
    return uattn


def _ids(kind, T, V, seed=0):
    g = inputs.rng(311, T, V, seed=seed)
    if kind == "uniform":
        ids = g.integers(0, V, T)
    elif kind == "zipf":
        ids = np.minimum(np.exp(g.random(T) * np.log(V)).astype(np.int64) - 1, V - 1)
    elif kind == "one":
        ids = np.full(T, V // 2)
    elif kind == "few":
        ids = g.integers(0, min(3, V), T) * ((V - 1) // max(1, min(3, V) - 1))
    elif kind == "sorted":
        ids = np.sort(g.integers(0, V, T))
    else:  # nothing to add: padding and ids past the table
        ids = np.where(g.random(T) < 0.5, -1 - g.integers(0, 5, T), V + g.integers(0, 5, T))
    if kind in ("uniform", "zipf"):
        ids = np.where(g.random(T) < 0.1, g.choice([-1, V, -(2 ** 31), 2 ** 31 - 1], T), ids)
    return ids.astype(np.int32)


def _strided(bits, extra=16):
    """The same rows in a buffer with `extra` more columns (filled with NaN)."""
    buf = np.full((bits.shape[0], bits.shape[1] + extra), 0x7FC0, dtype=np.uint16)
    buf[:, :bits.shape[1]] = bits
    return gu.dev(buf)[:, :bits.shape[1]]


@pytest.mark.parametrize("T,V,H,scale", [(1, 7, 8, 1.0), (5, 1000, 64, 8.0), (300, 32000, 1024, 32.0), (77, 50257, 2056, 0.3),
                                         (129, 128, 4096, 1.0)])
def test_lookup_matches_oracle(ua, T, V, H, scale):
    import torch
    table = inputs.normal_bf16((V, H), 0.02, 312, V, H)
    ids = _ids("uniform", T, V)
    want = oracle.embedding_fp64(ids, oracle.bf16_to_f64(table), scale)
    out = torch.full((T + 1, H + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    for tab in (gu.dev(table), _strided(table)):
        got = gu.host_f64(ua.embedding(gu.dev_i32(ids), tab, scale=scale, out=out[:T, :H]))
        ok = ~np.isnan(want)
        assert np.array_equal(np.isnan(got), ~ok)
        assert np.all(np.abs(got - want)[ok] <= (0.0 if scale in (1.0, 8.0, 32.0) else HALF + U) * np.abs(want[ok]))
    assert bool((out[T] == 7.0).all()) and bool((out[:, H:] == 7.0).all())


GRADS = [(1, 5, 8, "uniform"), (2, 1, 64, "one"), (64, 9, 512, "one"), (65, 9, 520, "one"), (1000, 9, 64, "few"),
         (300, 2000, 1024, "zipf"), (4095, 300, 64, "zipf"), (4097, 151936, 64, "uniform"), (9000, 1000, 72, "zipf"),
         (20000, 50257, 32, "zipf"), (8200, 40, 1032, "one"), (5000, 70000, 128, "sorted"), (777, 50, 64, "nothing"),
         (128, 513, 4096, "zipf"), (3000, 262145, 16, "uniform"), (16385, 511, 8, "uniform"), (16384, 512, 8, "few")]


@pytest.mark.parametrize("T,V,H,kind", GRADS)
@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_matches_oracle(ua, T, V, H, kind, fp32, accumulate):
    import torch
    dout = inputs.normal_bf16((T, H), 1.0, 313, T, H)
    ids = _ids(kind, T, V)
    scale = 0.7
    base = inputs.normal_bf16((V, H), 1.0, 314, V, H)
    want, mag, count = oracle.embedding_backward_fp64(oracle.bf16_to_f64(dout), ids, V, scale,
                                                      oracle.bf16_to_f64(base) if accumulate else None)
    grad = gu.dev(base)
    grad = grad.float() if fp32 else grad
    wide = torch.full((V, H + 8), 3.0, dtype=grad.dtype, device="cuda")   # rows of a wider buffer, the rest left alone
    wide[:, :H] = grad
    got = ua.embedding_backward(_strided(dout), gu.dev_i32(ids), V, scale=scale, grad=wide[:, :H], accumulate=accumulate)
    assert bool((wide[:, H:] == 3.0).all())
    have = got.double().cpu().numpy()
    # a run's tokens one after another in pieces, then the pieces: no more roundings than tokens, and two at the end
    bound = (count[:, None] + 2) * U * mag + (0.0 if fp32 else 1.0) * HALF * np.abs(want)
    assert np.all(np.abs(have - want) <= bound)
    untouched = count == 0
    assert np.array_equal(have[untouched], want[untouched])


@pytest.mark.parametrize("T,V,H", [(524288, 151936, 8), (524289, 777, 16), (1500000, 300000, 8), (3000000, 3, 8)])
def test_many_tokens(ua, T, V, H):
    """The tiles' counts summed by a launch of their own, and runs of a million tokens; fp64 sums on the GPU."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    ids = torch.randint(-1, V + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    dout = torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16)
    got = ua.embedding_backward(dout, ids, V)
    ok = (ids >= 0) & (ids < V)
    at, x = ids[ok].long(), dout[ok].double()
    want = torch.zeros((V, H), dtype=torch.float64, device="cuda").index_add_(0, at, x)
    mag = torch.zeros((V, H), dtype=torch.float64, device="cuda").index_add_(0, at, x.abs())
    count = torch.bincount(at, minlength=V)[:, None]
    # a piece's 32 tokens, then the pieces one after another, and the scale
    assert bool(((got.double() - want).abs() <= (34 + count / 32) * U * mag).all())
    assert torch.equal(got, ua.embedding_backward(dout, ids, V))


@pytest.mark.parametrize("T,V,H", [(700, 50, 256), (6000, 200, 64), (30000, 3000, 64)])
def test_rows_depend_on_their_own_tokens_alone(ua, T, V, H):
    """Other tokens put between, and calls in a row: the same bits for an entry's row."""
    import torch
    dout = gu.dev(inputs.normal_bf16((T, H), 1.0, 315))
    ids = _ids("zipf", T, V)
    first = ua.embedding_backward(dout, gu.dev_i32(ids), V)
    assert torch.equal(first, ua.embedding_backward(dout, gu.dev_i32(ids), V))
    keep = np.flatnonzero(ids % 3 == 1)
    part = ua.embedding_backward(dout[torch.from_numpy(keep).cuda()].contiguous(), gu.dev_i32(ids[keep]), V)
    assert torch.equal(part[1::3], first[1::3]) and not part[0::3].any()


def test_no_tokens(ua):
    import torch
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    g = torch.full((5, 64), 2.0, device="cuda")
    assert bool((ua.embedding_backward(e, ids, 5, grad=g, accumulate=True) == 2.0).all())
    assert not ua.embedding_backward(e, ids, 5, grad=g).any()
    assert ua.embedding(ids, torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda")).shape == (0, 64)


@pytest.mark.parametrize("T", [3000, 20000])
def test_captured_and_replayed(ua, T):
    """Two graphs with one workspace each, replayed in turn between eager calls on a third."""
    import torch
    V, H = 5000, 128
    outs, graphs, sets = [], [], []
    for i in range(2):
        dout, ids = gu.dev(inputs.normal_bf16((T, H), 1.0, 316, i)), gu.dev_i32(_ids("zipf", T, V, seed=i))
        table = gu.dev(inputs.normal_bf16((V, H), 1.0, 317, i))
        ua.embedding_backward(dout, ids, V)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            rows = ua.embedding(ids, table)
            grad = ua.embedding_backward(dout, ids, V)
        outs.append((rows, grad))
        graphs.append(g)
        sets.append((dout, ids, table))
    for rep in range(3):
        for i, (dout, ids, table) in enumerate(sets):
            ids.copy_(gu.dev_i32(_ids("zipf", T, V, seed=10 * rep + i)))
            dout.mul_(-0.5)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (rows, grad), (dout, ids, table) in zip(outs, sets):
            assert torch.equal(grad, ua.embedding_backward(dout, ids, V)) and torch.equal(
                rows.view(torch.int16), ua.embedding(ids, table).view(torch.int16))


def test_streams(ua):
    import torch
    sets = [(gu.dev(inputs.normal_bf16((9000, 256), 1.0, 318, i)), gu.dev_i32(_ids("zipf", 9000, 3000, seed=i))) for i in range(2)]
    want = [ua.embedding_backward(d, ids, 3000) for d, ids in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        got = [ua.embedding_backward(d, ids, 3000, stream=st) for (d, ids), st in zip(sets, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_past_2_31_elements(ua):
    """A table and a gradient whose last rows lie behind 2^32 bytes."""
    import torch
    V, H = 300000, 8192
    table = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    last = gu.dev(inputs.normal_bf16((3, H), 1.0, 319))
    table[V - 3:] = last
    ids = gu.dev_i32([V - 1, 0, V - 3, V - 2, V - 1])
    out = ua.embedding(ids, table)
    assert torch.equal(out[[0, 2, 3, 4]], last[[2, 0, 1, 2]]) and not out[1].any()
    ua.embedding_backward(out, ids, V, grad=table)
    assert torch.equal(table[V - 2], last[1]) and torch.equal(table[V - 1], (2 * last[2].float()).to(torch.bfloat16))
    assert not table[:V - 3].any()


@pytest.mark.parametrize("fp32", [True, False])
def test_widest_rows(ua, fp32):
    """The most columns there may be, small whole numbers: sums up to 70 * 3 are exact in fp32 and in bf16."""
    import torch
    T, V, H = 70, 3, 1 << 20
    ids = gu.dev_i32(inputs.rng(356, T).integers(-1, V, T).astype(np.int32))
    table = torch.arange(V * H, device="cuda").remainder(7).sub(3).to(torch.bfloat16).reshape(V, H)
    out = ua.embedding(ids, table)
    for t in range(T):
        assert torch.equal(out[t], table[ids[t]] if ids[t] >= 0 else torch.zeros_like(out[t]))
    grad = ua.embedding_backward(out, ids, V, dtype=torch.float32 if fp32 else torch.bfloat16)
    want = torch.stack([table[v].float() * int((ids == v).sum()) for v in range(V)])
    assert torch.equal(grad.float(), want if fp32 else want.to(torch.bfloat16).float())


def test_validation(ua, monkeypatch):
    import torch
    monkeypatch.setenv("UATTN_VALIDATE", "1")
    t = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    assert ua.embedding(gu.dev_i32([0, 3, -1]), t).shape == (3, 64)
    assert ua.embedding_backward(t, gu.dev_i32([0, 3, -1, 2]), 4).shape == (4, 64)
    with pytest.raises(ua.UattnError):
        ua.embedding(gu.dev_i32([0, 4]), t)
    with pytest.raises(ua.UattnError):
        ua.embedding_backward(t, gu.dev_i32([0, 3, 4, 2]), 4)


def test_binding_refuses(ua):
    import torch
    t = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    for f in (lambda: ua.embedding(ids.long(), t), lambda: ua.embedding(ids, t.float()), lambda: ua.embedding(ids[:, None], t),
              lambda: ua.embedding(ids, t, out=torch.empty_like(t)[:2]), lambda: ua.embedding_backward(t, ids[:2], 4),
              lambda: ua.embedding_backward(t, ids, 4, accumulate=True),
              lambda: ua.embedding_backward(t, ids, 5, grad=torch.zeros((4, 64), device="cuda")),
              lambda: ua.embedding_backward(t, ids, 4, dtype=torch.float16)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ua.embedding(ids, t[:, :12].contiguous()), lambda: ua.embedding(ids, t, scale=float("nan")),
              lambda: ua.embedding_backward(t, ids, 0), lambda: ua.embedding(ids, t[:, 4:60]),
              lambda: ua.embedding_backward(t, ids, 4, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ua.UattnError):
            f()


@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("accumulate", [False, True])
def test_large_gradient(ua, fp32, accumulate):
    """256 MB of rows: read past the caches, added to a table or written whole; fp64 sums on the GPU."""
    import torch
    T, V, H = 65536, 20000, 2048
    g = torch.Generator(device="cuda")
    g.manual_seed(323)
    dout = torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16)
    ids = gu.dev_i32(_ids("zipf", T, V))
    base = torch.randn((V, H), generator=g, device="cuda").to(torch.float32 if fp32 else torch.bfloat16)
    got = ua.embedding_backward(dout, ids, V, scale=0.5, grad=base.clone(), accumulate=accumulate)
    ok = (ids >= 0) & (ids < V)
    at, x = ids[ok].long(), dout[ok].double() * 0.5
    start = base.double() if accumulate else torch.zeros((V, H), dtype=torch.float64, device="cuda")
    want = start.clone().index_add_(0, at, x)
    mag = start.abs().index_add_(0, at, x.abs())
    count = torch.bincount(at, minlength=V)[:, None]
    # a piece's 32 tokens, then the pieces one after another, the sum with the table's value; a half step of the result's type
    bound = (34 + count / 32) * U * mag + (0.0 if fp32 else HALF) * want.abs()
    assert bool(((got.double() - want).abs() <= bound).all())
    assert torch.equal(got[count[:, 0] == 0].double(), start[count[:, 0] == 0])


def test_large_lookup(ua):
    """64 MB of rows: written past the caches, into rows of a wider buffer."""
    import torch
    T, V, H = 8300, 5000, 4096
    table = torch.randn((V, H), device="cuda").to(torch.bfloat16)
    ids = gu.dev_i32(_ids("uniform", T, V))
    out = torch.full((T, H + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ua.embedding(ids, table, out=out[:, :H])
    at = ids.long()
    known = (at >= 0) & (at < V)
    assert torch.equal(out[known, :H], table[at[known]]) and not out[at < 0, :H].any() and bool(torch.isnan(out[at >= V, :H]).all())
    assert bool((out[:, H:] == 7.0).all())
