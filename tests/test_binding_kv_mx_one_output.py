"""One of the two outputs of the rows read back or rounded given, without a GPU: the other is made alike."""
import pytest
import torch

BF16, I32, U8 = torch.bfloat16, torch.int32, torch.uint8


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def t(shape, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    """{name: (k, v) -> (the outputs, the stride that the library got)} for three tokens of two heads of 64."""
    from paper_2609_35140_amd import uattn
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append(args) or 0

    monkeypatch.setattr(uattn, "_load", Library)
    monkeypatch.setattr(uattn, "_elsewhere", lambda device, stream: None)
    monkeypatch.setattr(uattn, "_stream_on", lambda device: 0)
    cache = tuple(t((4, 2, 16, w), U8) for w in (64, 2, 32, 2))

    def read(k, v, n=3):
        out = uattn.kv_read_mx(*cache, t((2, 4), I32), t((n,), I32), t((n,), I32), k_out=k, v_out=v)
        return out, seen[-1][-2]

    def round_(k, v, n=3):
        return uattn.kv_round_mx(t((n, 2, 64)), t((n, 2, 64)), 8, 4, k_out=k, v_out=v), seen[-1][-2]

    return {"read": read, "round": round_}


@pytest.mark.parametrize("name", ["read", "round"])
@pytest.mark.parametrize("which", [0, 1])
def test_a_strided_one(calls, name, which):
    given = t((3, 8, 64))[:, 4:6]
    outs = [None, None]
    outs[which] = given
    got, stride = calls[name](*outs)
    assert stride == 512 and got[which] is given
    assert got[1 - which].shape == (3, 2, 64) and got[1 - which].stride() == (512, 64, 1) and got[1 - which].dtype is BF16


@pytest.mark.parametrize("name", ["read", "round"])
@pytest.mark.parametrize("which", [0, 1])
def test_contiguous_ones_and_one_token(calls, name, which):
    for given, n in ((t((3, 2, 64)), 3), (t((1, 2, 64)), 1), (t((1, 8, 64))[:, 4:6], 1), (t((0, 8, 64))[:, 4:6], 0)):
        outs = [None, None]
        outs[which] = given
        got, stride = calls[name](*outs, n)
        assert stride == 128 and got[1 - which].shape == (n, 2, 64)


@pytest.mark.parametrize("name", ["read", "round"])
@pytest.mark.parametrize("which", [0, 1])
def test_what_does_not_fit_is_refused(calls, name, which):
    for given in (t((4, 2, 64)), t((3, 2, 128)), t((3, 3, 64)), t((3, 128)), t((3, 8, 64))[:, ::2][:, :2], t((3, 2, 64), torch.float32)):
        outs = [None, None]
        outs[which] = given
        with pytest.raises(ValueError):
            calls[name](*outs)
