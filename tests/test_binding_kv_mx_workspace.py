"""The workspace that the two decodes may share, without a GPU: a library that does to it what the kernels do (partials at its
end; the bf16 decode expects its counters at the start to be zero)."""
import ctypes
import os

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
def ua(monkeypatch):
    from paper_2609_35140_amd import uattn
    if not os.path.exists(uattn.LIB_PATH):
        from paper_2609_35140_amd import build
        build.build()
    real = uattn.lib()

    class Library:
        def __getattr__(self, name):
            return getattr(real, name)  # sizes

        def uattn_decode_mx(self, *a):
            B, most, hq, hkv, d, ws, size = a[9], *a[13:17], a[20], a[21]
            need = real.uattn_decode_mx_workspace_bytes(B, most, hq, hkv, d)
            assert need <= size
            if need:
                ctypes.memset(ws + (size & ~15) - need, 0xFF, need)
            return 0

        def uattn_decode(self, *a):
            B, most, hq, d, ws, size = a[5], a[9], a[10], a[12], a[16], a[17]
            if real.uattn_decode_workspace_bytes(B, most, hq, d):
                counters = ctypes.string_at(ws, uattn.counter_bytes(B, hq))
                assert not any(counters), "a decode's counters are not zero"
                partials = real.uattn_decode_workspace_bytes(B, most, hq, d) - len(counters)
                ctypes.memset(ws + (size & ~15) - partials, 0xFF, partials)
            return 0

    monkeypatch.setattr(uattn, "_load", Library)
    monkeypatch.setattr(uattn, "_elsewhere", lambda device, stream: None)
    monkeypatch.setattr(uattn, "_stream_on", lambda device: 0)
    monkeypatch.setattr(uattn, "_stream", lambda stream: 0)
    return uattn


def _mx(ua, ws, B, most, hq=8, hkv=2, d=128):
    cache = tuple(t((4, hkv, 16, w), U8) for w in (d, d // 32, d // 2, d // 32))
    ua.decode_mx(t((B, hq, d)), *cache, t((B, -(-most // 16)), I32), t((B,), I32), most, workspace=ws)


def _bf16(ua, ws, B, most, hq=8, hkv=2, d=128):
    pages = t((4, hkv, 16, d))
    ua.decode(t((B, hq, d)), pages, pages, t((B, -(-most // 16)), I32), t((B,), I32), most, workspace=ws)


def _workspace(ua, size):
    ws = torch.zeros(size, dtype=U8).as_subclass(OnGpu)
    ws._uattn_zero_prefix = size  # as new_workspace leaves it
    return ws


@pytest.mark.parametrize("extra", [0, 16, 100, 300, 5000])
def test_a_workspace_of_the_mx_decodes_own_size(ua, extra):
    """Large enough for the partials, too small for a bf16 decode of these sizes: the partials reach the counters of a smaller one."""
    need = ua.decode_mx_workspace_bytes(2, 5000, 8, 2, 128)
    assert need > 0
    ws = _workspace(ua, need + extra)
    _bf16(ua, ws, 1, 600)
    for _ in range(2):
        _mx(ua, ws, 2, 5000)
        _bf16(ua, ws, 1, 600)
        _bf16(ua, ws, 2, 300)


def test_a_larger_batch_behind_the_mx_decode(ua):
    """The bf16 decode's counters past those that the mx decode's sizes would have."""
    ws = _workspace(ua, ua.decode_workspace_bytes(3, 20000, 8, 128))
    _mx(ua, ws, 3, 20000)
    _bf16(ua, ws, 60, 500)


def test_counters_that_the_partials_leave_alone_stay_known(ua):
    """Nothing is cleared again where a call cannot have reached the counters."""
    size = ua.decode_workspace_bytes(3, 5000, 8, 128)
    ws = _workspace(ua, size)
    _mx(ua, ws, 3, 5000)
    assert ws._uattn_zero_prefix == ua.counter_bytes(3, 8)
    _mx(ua, ws, 3, 2000)     # folded in LDS: no partials
    assert ws._uattn_zero_prefix == ua.counter_bytes(3, 8)
    ws = _workspace(ua, 4 * size)
    _mx(ua, ws, 3, 5000)
    assert ws._uattn_zero_prefix >= 3 * size
