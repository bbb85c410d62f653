"""The binding's calls for a cache in 8 or 4 bits, without a GPU: which sizes, widths and strides reach the library.

Tensors stand here without memory ("meta" tensors that say they are on a GPU); the library is one that takes nothing.
"""
import pytest
import torch

BF16, I32, U8 = torch.bfloat16, torch.int32, torch.uint8
WRAPS = 2 ** 32 + 64  # 64 without the high bits


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def t(shape, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu)


@pytest.fixture
def ua(monkeypatch):
    from paper_2609_35140_amd import uattn

    class Library:
        def __getattr__(self, name):
            if name.endswith("workspace_bytes"):
                return lambda *sizes: 16
            return lambda *args: pytest.fail(f"{name} was reached with {args}")

    monkeypatch.setattr(uattn, "_load", Library)
    monkeypatch.setattr(uattn, "_elsewhere", lambda device, stream: None)
    monkeypatch.setattr(uattn, "_stream_on", lambda device: 0)
    uattn._decode_mx_need.cache_clear()
    yield uattn
    uattn._decode_mx_need.cache_clear()


def _cache(P=4, K=2, page=16, D=64, bits=(8, 4)):
    return tuple(t((P, K, page, w), U8) for w in (D * bits[0] // 8, D // 32, D * bits[1] // 8, D // 32))


def _write(N=3, B=2, maxp=4, **kw):
    c = _cache(**kw)
    rows = t((N, c[1].shape[1], c[1].shape[3] * 32))
    return lambda ua: ua.kv_write_mx(rows, rows, t((B, maxp), I32), t((N,), I32), t((N,), I32), *c)


def _read(N=3, B=2, maxp=4, **kw):
    return lambda ua: ua.kv_read_mx(*_cache(**kw), t((B, maxp), I32), t((N,), I32), t((N,), I32))


def _round(N=3, K=2, D=64):
    return lambda ua: ua.kv_round_mx(t((N, K, D)), t((N, K, D)), 8, 4)


def _decode(B=2, H=4, maxp=4, most=40, **kw):
    c = _cache(**kw)
    return lambda ua: ua.decode_mx(t((B, H, c[1].shape[3] * 32)), *c, t((B, maxp), I32), t((B,), I32), most)


@pytest.mark.parametrize("call", [
    _write(N=WRAPS), _write(B=WRAPS), _write(maxp=WRAPS), _write(P=WRAPS), _write(K=WRAPS), _write(page=2 ** 32 + 16),
    _read(N=WRAPS), _read(B=2 ** 31), _read(maxp=WRAPS), _read(P=WRAPS), _round(N=WRAPS), _round(K=WRAPS),
    _decode(B=WRAPS), _decode(H=WRAPS), _decode(maxp=WRAPS), _decode(most=WRAPS), _decode(most=-WRAPS), _decode(P=WRAPS),
])
def test_sizes_past_32_bits_are_refused(ua, call):
    with pytest.raises(ValueError, match="2\\^31"):
        call(ua)


@pytest.mark.parametrize("bits", [(8, 8), (4, 4), (8, 4), (4, 8)])
def test_bits_follow_from_the_widths(ua, monkeypatch, bits):
    seen = {}

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.update({name: args}) or (16 if name.endswith("bytes") else 0)

    monkeypatch.setattr(ua, "_load", Library)
    ua._decode_mx_need.cache_clear()
    for D in (64, 128):
        for call in (_write(D=D, bits=bits), _read(D=D, bits=bits), _decode(D=D, bits=bits, page=32)):
            call(ua)
        assert seen["uattn_kv_write_mx"][6:15] == (3, 2, 4, 16, 4, 2, D, *bits)
        assert seen["uattn_kv_read_mx"][4:6] == bits and seen["uattn_kv_read_mx"][9:16] == (3, 2, 4, 16, 4, 2, D)
        assert seen["uattn_decode_mx"][5:7] == bits and seen["uattn_decode_mx"][9:17] == (2, 4, 32, 4, 40, 4, 2, D)


def test_strides(ua, monkeypatch):
    """Rows inside the projection's pass their distance on; one token may have any."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append(args) or 0

    monkeypatch.setattr(ua, "_load", Library)
    fused = t((5, 8, 64))
    ua.kv_round_mx(fused[:, 4:6], fused[:, 6:], k_out=fused[:, 4:6], v_out=fused[:, 6:])
    assert seen[-1][2] == 512 and seen[-1][-2] == 512
    ua.kv_round_mx(fused[:1, 4:6], fused[:1, 6:], k_out=t((1, 2, 64)), v_out=t((1, 2, 64)))
    assert seen[-1][2] == 128
    for k, v in ((fused[:, ::2], fused[:, ::2]), (fused[:, :2], t((5, 2, 64))), (fused[..., :32], fused[..., 32:]), (fused, fused[:4])):
        with pytest.raises(ValueError):
            ua.kv_round_mx(k, v)
