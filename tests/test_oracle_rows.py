"""Pins of the row-wise operators' oracles: differences, automatic differentiation in float64, closed forms."""
import math

import numpy as np
import pytest

import oracle


def _rand(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def _parts(post, gate, T=5, H=16):
    return dict(pre=1 + 0.1 * _rand(1, H), x=_rand(2, T, H), post=1 + 0.1 * _rand(3, H) if post else None,
                gate=None if gate == "none" else _rand(4, H) if gate == "shared" else _rand(4, T, H), scale=0.5, eps=1e-5)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "shared", "token"])
def test_norm_gradients_are_differences_of_the_forward(post, gate):
    """Of L = sum dy y(s) + sum dres s with s the forward's sum (fp64, not rounded): every input's central difference."""
    k = _parts(post, gate)
    res, dy, dres = _rand(5, 5, 16), _rand(6, 5, 16), _rand(7, 5, 16)

    def loss(residual, **kw):
        (s, y), _ = oracle.residual_norm_fp64(residual, **kw)
        return (dy * y).sum() + (dres * s).sum()

    (s, _), _ = oracle.residual_norm_fp64(res, **k)
    val, mag = oracle.residual_norm_backward_fp64(dy, dres, s, **k)
    of = {"dresidual": None, "dx": "x", "dpre": "pre", "dpost": "post", "dgate": "gate"}
    for name, g in val.items():
        assert np.all(np.abs(g) <= mag[name] * (1 + 1e-12))
        src = res if of[name] is None else k[of[name]]
        num = np.zeros_like(src)
        for i in np.ndindex(src.shape):
            lo, hi = src.copy(), src.copy()
            lo[i] -= 1e-6
            hi[i] += 1e-6
            a, b = ((loss(v, **k) if of[name] is None else loss(res, **{**k, of[name]: v})) for v in (hi, lo))
            num[i] = (a - b) / 2e-6
        assert np.abs(num - g).max() < 1e-6, name
    assert ("dpost" in val) == post and ("dgate" in val) == (gate != "none")


def test_norm_closed_forms():
    h = np.full((1, 8), 3.0)
    (s, y), _ = oracle.residual_norm_fp64(h, pre=np.arange(8.0), eps=0.0)
    assert np.array_equal(s, h) and np.allclose(y[0], np.arange(8.0))
    (s, y), _ = oracle.residual_norm_fp64(h, x=np.full((1, 8), -2.0), gate=np.ones(8), scale=0.5)
    assert np.array_equal(s, np.full((1, 8), 2.0)) and y is None
    # y does not change with the length of s: the gradient is orthogonal to s
    val, _ = oracle.residual_norm_backward_fp64(_rand(1, 2, 8), None, _rand(2, 2, 8), pre=_rand(3, 8), eps=0.0, block=False)
    assert np.abs((val["dresidual"] * _rand(2, 2, 8)).sum(-1)).max() < 1e-12


def test_embedding_oracle():
    table = _rand(1, 5, 8)
    out = oracle.embedding_fp64([4, -1, 0, 5], table, 2.0)
    assert np.array_equal(out[0], 2 * table[4]) and not out[1].any() and np.isnan(out[3]).all()
    dout = _rand(2, 6, 8)
    g, mag, n = oracle.embedding_backward_fp64(dout, [1, 1, -3, 4, 1, 5], 5, 0.5)
    assert np.allclose(g[1], 0.5 * (dout[0] + dout[1] + dout[4])) and n.tolist() == [0, 3, 0, 0, 1]
    assert not g[0].any() and np.all(mag >= np.abs(g))
    # <grad, table> = <dout, lookup> for ids inside the table
    ids = [0, 3, 3, 2, 1, 0]
    g, _, _ = oracle.embedding_backward_fp64(dout, ids, 5, 0.5)
    assert abs((g * table).sum() - (dout * oracle.embedding_fp64(ids, table, 0.5)).sum()) < 1e-12


def test_logits_oracle_by_hand():
    z = np.array([[2.0, -2.0, 4.0, 0.0, 1.0, 3.0]])
    kw = dict(tokens=np.array([0, 1, 2, 2, 9, -1]), history=[[0, 2, 6]], penalties=[[2.0, 0.5, 0.25]])
    out, _ = oracle.logits_process_fp64(z, **kw)
    assert out[0].tolist() == [1.0, -4.0, 4.0 / 2 - 0.5 * 2 - 0.25, 0.0, 1.0, 3.0]
    out, _ = oracle.logits_process_fp64(z, **kw, bias_ids=[4, 4, 7], bias_values=[9.0, -1.0, 5.0], bias_rows=[[0, 3]],
                                        mask=np.array([[0b011111]]))
    assert out[0].tolist() == [1.0, -4.0, 0.75, 0.0, 0.0, -math.inf]
    d = oracle.logits_process_backward_fp64(np.ones((1, 6)), z, **kw, mask=np.array([[0b011111]]), mask_rows=[0])
    assert d[0].tolist() == [0.5, 2.0, 0.5, 1.0, 1.0, 0.0]
    d = oracle.logits_process_backward_fp64(np.ones((1, 6)), z, mask=np.array([[0]]), mask_rows=[-1])
    assert d[0].tolist() == [1.0] * 6


def test_logits_gradient_is_the_difference():
    z = _rand(3, 3, 11) * 2
    kw = dict(tokens=np.random.default_rng(4).integers(0, 11, 30), history=[[0, 5, 9], [3, 3, 3], [10, 20, 30]],
              penalties=[[1.3, 0.2, 0.1], [1.5, 1, 1], [0.8, 0.0, 0.3]])
    d = _rand(5, 3, 11)
    g = oracle.logits_process_backward_fp64(d, z, **kw)
    num = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        hi, lo = z.copy(), z.copy()
        hi[i] += 1e-6
        lo[i] -= 1e-6
        num[i] = ((oracle.logits_process_fp64(hi, **kw)[0] - oracle.logits_process_fp64(lo, **kw)[0]) * d).sum() / 2e-6
    assert np.abs(num - g).max() < 1e-6


def test_logprob_gradient_oracle():
    import torch
    z = _rand(6, 4, 13) * 3
    z[2, 5] = -np.inf
    tg, g, it = [0, 12, 3, 7], np.array([0.5, -2.0, 1.0, 0.0]), 1.25
    x = torch.tensor(z, requires_grad=True)
    lp = torch.log_softmax(x * it, 1)[torch.arange(4), torch.tensor(tg)]
    (lp * torch.tensor(g)).sum().backward()
    out, err = oracle.logprob_backward_fp64(z, tg, g, it)
    assert np.abs(out - x.grad.numpy()).max() < 1e-14 and not out[3].any() and np.all(err < 1e-4)
    assert np.abs(out[:3].sum(1)).max() < 1e-14 and out[2, 5] == 0
    # a nearly certain target keeps its digits: 1 - p of two entries 60 apart is exp(-60)
    out, _ = oracle.logprob_backward_fp64(np.array([[60.0, 0.0]]), [0], [1.0])
    assert abs(out[0, 0] / math.exp(-60) - 1) < 1e-12
    assert np.isnan(oracle.logprob_backward_fp64(z, [13, 0, 0, 0], [1, 1, 1, 1])[0][0]).all()


# Planted mistakes: each has to fall outside what the GPU tests allow (2^-8 of the value, 2^-15 of its terms).
@pytest.mark.parametrize("mistake", ["eps", "mean", "weight", "gate", "second"])
def test_planted_norm_mistakes_are_seen(mistake):
    T, H = 6, 64
    k = dict(pre=1 + 0.1 * _rand(1, H), post=1 + 0.1 * _rand(2, H), gate=_rand(3, H), x=0.05 * _rand(4, T, H), scale=0.5, eps=1e-2)
    res = _rand(5, T, H)
    (s, y), (_, size) = oracle.residual_norm_fp64(res, **k)
    bad = dict(k)
    if mistake == "eps":
        bad["eps"] = 1e-6
    elif mistake == "mean":
        bad["pre"] = k["pre"] * math.sqrt((H - 1) / H)
    elif mistake == "weight":
        bad["pre"] = k["post"]
    elif mistake == "gate":
        bad["gate"] = None
    else:
        bad["post"] = None
    (_, other), _ = oracle.residual_norm_fp64(res, **bad)
    assert np.any(np.abs(other - y) > 2.0 ** -8 * np.abs(y) + 2.0 ** -15 * size)
