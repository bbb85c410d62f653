"""Argument checks of the row-wise entry points, on the host before anything is launched, and their workspace sizes."""
import ctypes
import os

import pytest

P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_2609_35140_amd import uattn
    if not os.path.exists(uattn.LIB_PATH):
        from paper_2609_35140_amd import build
        build.build()
    return uattn.lib()


def _call(fn, defaults, kw):
    unknown = set(kw) - set(defaults)
    assert not unknown, unknown
    return fn(*{**defaults, **kw}.values())


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), 1), (dict(H=0), 1), (dict(H=12), 2), (dict(H=16392), 2), (dict(scale=NAN), 1), (dict(scale=INF), 1),
    (dict(eps=-1.0), 1), (dict(eps=NAN), 1), (dict(eps=INF), 1), (dict(gs=63), 1), (dict(gs=-64), 1), (dict(res=None), 1),
    (dict(y=None), 1), (dict(pre=None), 1), (dict(x=None), 1), (dict(ro=None), 1), (dict(x=None, ro=None), 1),
    (dict(x=None, ro=None, post=None, gate=None, y=None, pre=None), 1), (dict(x=P(24)), 1), (dict(gate=P(24)), 1),
    (dict(y=P(18)), 1), (dict(T=0), 0), (dict(T=0, res=None), 0),
])
def test_residual_norm(lib, kw, code):
    d = dict(x=P(16), post=P(16), gate=P(16), gs=0, scale=1.0, res=P(16), pre=P(16), eps=1e-6, T=4, H=64, ro=P(16), y=P(16),
             stream=None)
    assert _call(lib.uattn_residual_norm, d, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), 1), (dict(H=12), 2), (dict(H=16392), 2), (dict(scale=NAN), 1), (dict(eps=-1.0), 1), (dict(gs=8), 1),
    (dict(dpre=None), 1), (dict(pre=None), 1), (dict(dy=None), 1), (dict(dpost=None), 1), (dict(dgate=None), 1),
    (dict(post=None), 1), (dict(gate=None), 1), (dict(h=None), 1), (dict(dres=None), 1), (dict(x=None), 1), (dict(dx=None), 1),
    (dict(dy=None, pre=None, dpre=None, dro=None), 1), (dict(dro=P(24)), 1), (dict(dpre=P(24)), 1),
    (dict(ws=None), 3), (dict(wsb=100), 3), (dict(ws=P(24)), 3),
])
def test_residual_norm_backward(lib, kw, code):
    d = dict(dy=P(16), dro=P(16), h=P(16), pre=P(16), x=P(16), post=P(16), gate=P(16), gs=0, scale=1.0, eps=1e-6, T=4, H=64,
             dres=P(16), dx=P(16), dpre=P(16), dpost=P(16), dgate=P(16), ws=P(16), wsb=1 << 20, stream=None)
    assert _call(lib.uattn_residual_norm_backward, d, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(H=0), 1), (dict(H=12), 1), (dict(scale=NAN), 1), (dict(ts=60), 1), (dict(ts=68), 1),
    (dict(os=32), 1), (dict(ids=None), 1), (dict(table=None), 1), (dict(out=None), 1), (dict(table=P(24)), 1),
    (dict(out=P(24)), 1), (dict(T=0), 0), (dict(H=(1 << 20) + 8, ts=1 << 21, os=1 << 21), 2),
])
def test_embedding(lib, kw, code):
    d = dict(ids=P(16), table=P(16), ts=64, scale=1.0, T=4, V=10, H=64, out=P(16), os=64, stream=None)
    assert _call(lib.uattn_embedding, d, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(V=-5), 1), (dict(H=12), 1), (dict(scale=INF), 1), (dict(ds=60), 1), (dict(ds=68), 1),
    (dict(gs=60), 1), (dict(gs=66), 1), (dict(gs=68, fp32=0), 1), (dict(fp32=2), 1), (dict(acc=-1), 1), (dict(grad=None), 1),
    (dict(dout=None), 1), (dict(ids=None), 1), (dict(dout=P(24)), 1), (dict(grad=P(24)), 1), (dict(T=(1 << 30) + 1), 2),
    (dict(ws=None), 3), (dict(wsb=100), 3), (dict(ws=P(24)), 3), (dict(T=0, acc=1), 0),
    (dict(H=(1 << 20) + 8, ds=1 << 21, gs=1 << 21), 2),
])
def test_embedding_backward(lib, kw, code):
    d = dict(dout=P(16), ds=64, ids=P(16), scale=1.0, T=4, V=10, H=64, grad=P(16), gs=64, fp32=1, acc=0, ws=P(16), wsb=1 << 20,
             stream=None)
    assert _call(lib.uattn_embedding_backward, d, kw) == code


LOGITS = [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(ls=96), 1), (dict(ls=108), 1), (dict(os=96), 1), (dict(os=108), 1),
    (dict(N=-1), 1), (dict(tok=None), 1), (dict(hist=None), 1), (dict(pen=None), 1), (dict(K=-1), 1), (dict(ms=3), 1),
    (dict(mr=None), 1), (dict(z=None), 1), (dict(out=None), 1), (dict(z=P(24)), 1), (dict(out=P(24)), 1), (dict(T=0), 0),
    (dict(T=0, z=None, out=None), 0), (dict(N=(1 << 30) + 1), 2),
]


@pytest.mark.parametrize("kw,code", LOGITS + [(dict(M=-1), 1), (dict(bi=None), 1), (dict(bv=None), 1), (dict(M=(1 << 30) + 1), 2)])
def test_logits_process(lib, kw, code):
    d = dict(z=P(16), ls=104, T=4, V=100, tok=P(16), N=9, hist=P(16), pen=P(16), bi=P(16), bv=P(16), M=2, br=P(16), mask=P(16),
             ms=4, K=2, mr=P(16), out=P(16), os=104, stream=None)
    assert _call(lib.uattn_logits_process, d, kw) == code


@pytest.mark.parametrize("kw,code", LOGITS + [(dict(d=None), 1), (dict(d=P(24)), 1), (dict(ds=96), 1), (dict(ds=108), 1)])
def test_logits_process_backward(lib, kw, code):
    d = dict(d=P(16), ds=104, z=P(16), ls=104, T=4, V=100, tok=P(16), N=9, hist=P(16), pen=P(16), mask=P(16), ms=4, K=2,
             mr=P(16), out=P(16), os=104, stream=None)
    assert _call(lib.uattn_logits_process_backward, d, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), 1), (dict(V=0), 1), (dict(ls=96), 1), (dict(ls=108), 1), (dict(os=96), 1), (dict(os=108), 1), (dict(it=0.0), 1),
    (dict(it=NAN), 1), (dict(it=INF), 1), (dict(it=3e38), 1), (dict(z=None), 1), (dict(tg=None), 1), (dict(dl=None), 1),
    (dict(out=None), 1), (dict(z=P(24)), 1), (dict(out=P(24)), 1), (dict(T=0), 0),
])
def test_logprob_backward(lib, kw, code):
    d = dict(z=P(16), ls=104, tg=P(16), dl=P(16), T=4, V=100, it=1.0, out=P(16), os=104, stream=None)
    assert _call(lib.uattn_logprob_backward, d, kw) == code


def test_workspace_bytes(lib):
    from paper_2609_35140_amd import uattn
    f, g = uattn.residual_norm_backward_workspace_bytes, uattn.embedding_backward_workspace_bytes
    assert f(0, 64) == f(-1, 64) == f(4, 12) == f(4, 1 << 20) == 0
    assert g(0, 64) == g(-1, 64) == g(4, 0) == g(4, (1 << 20) + 8) == 0
    # three sums of a group of rows each; they stop growing with the tokens
    assert f(1, 64) == 3 * 64 * 4 and f(100000, 4096) == f(1 << 30, 4096)
    # sorted keys and order, and for every 32 tokens two fp32 rows of partial sums
    assert 16 * 4096 + 2 * 128 * 1024 * 4 <= g(4096, 1024) <= 64 * 4096 + 2 * 128 * 1024 * 4 + (1 << 20)
    assert g(1 << 30, 8) > 1 << 32


def test_stream_of_another_gpu_is_refused():
    """The binding moves to the tensors' GPU, so a call for such a stream would run on another one than it names."""
    from paper_2609_35140_amd import uattn

    class Stream:
        cuda_stream, device_index = 5, 1

    with pytest.raises(ValueError, match="GPU 1"):
        uattn._elsewhere(0, Stream())


@pytest.mark.parametrize("handle", [0, 1])
def test_handle_of_the_default_stream(monkeypatch, handle):
    """0, and 1 by its other name, are the default stream's handles; torch would take 0 for no handle at all."""
    import torch
    from paper_2609_35140_amd import uattn

    class Default:
        cuda_stream = 0

        def __init__(self, device):
            self.device_index = device

    def external(*args, **kw):
        raise AssertionError("a handle of the default stream is no external stream")

    monkeypatch.setattr(torch.cuda, "default_stream", Default)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: stream)
    there = uattn._elsewhere(3, handle)
    assert isinstance(there, Default) and there.device_index == 3


def test_logprob_backward_in_place_is_refused(lib):
    """A workgroup's waves read the target's logit while others write: not in place, whatever the strides."""
    d = dict(z=P(16), ls=104, tg=P(16), dl=P(16), T=4, V=100, it=1.0, out=P(16), os=104, stream=None)
    assert _call(lib.uattn_logprob_backward, d, {}) == 1
    assert _call(lib.uattn_logprob_backward, d, dict(os=112)) == 1
    assert _call(lib.uattn_logprob_backward, d, dict(T=1)) == 1


def test_logits_in_place_with_another_stride_is_refused(lib):
    """Rows would be written over other rows, which other workgroups still read.  One row has no stride."""
    d = dict(z=P(16), ls=104, T=4, V=100, tok=P(16), N=9, hist=P(16), pen=P(16), bi=P(16), bv=P(16), M=2, br=P(16), mask=P(16),
             ms=4, K=2, mr=None, out=P(16), os=112, stream=None)
    assert _call(lib.uattn_logits_process, d, dict(K=4)) == 1
    d = dict(d=P(16), ds=104, z=P(32), ls=104, T=4, V=100, tok=P(16), N=9, hist=P(16), pen=P(16), mask=P(16), ms=4, K=4,
             mr=None, out=P(16), os=112, stream=None)
    assert _call(lib.uattn_logits_process_backward, d, {}) == 1
