"""Argument checks of the entry points for a cache in 8 or 4 bits, on the host before anything is launched."""
import ctypes
import os

import pytest

P = ctypes.c_void_p
INF, NAN = float("inf"), float("nan")


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


SHARED = [  # what every entry point with a cache refuses alike
    (dict(d=96), 2), (dict(page=8), 2), (dict(page=24), 2), (dict(page=0), 2), (dict(kb=16), 2), (dict(kb=0), 2), (dict(vb=5), 2),
    (dict(hkv=0), 1), (dict(B=-1), 1), (dict(maxp=-1), 1), (dict(np=-1), 1),
    (dict(kc=P(24)), 1), (dict(ks=P(24)), 1), (dict(vc=P(17)), 1), (dict(vs=P(20)), 1),
    (dict(kc=None), 1), (dict(ks=None), 1), (dict(vc=None), 1), (dict(vs=None), 1), (dict(bt=None), 1),
]
TOKENS = [(dict(N=-1), 1), (dict(st=127), 1), (dict(st=132), 1), (dict(st=-128), 1), (dict(hkv=65536, st=1 << 23), 2),
          (dict(seq=None), 1), (dict(pos=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(k=P(24)), 1), (dict(v=P(18)), 1),
          (dict(N=0), 0), (dict(N=0, k=None, v=None, kc=None, bt=None), 0)]


@pytest.mark.parametrize("kw,code", SHARED + TOKENS + [(dict(np=0), 0), (dict(B=0, bt=None), 0), (dict(maxp=0), 0)])
def test_write(lib, kw, code):
    d = dict(k=P(16), v=P(16), st=128, bt=P(16), seq=P(16), pos=P(16), N=4, B=2, maxp=4, page=16, np=8, hkv=2, d=64, kb=8, vb=4,
             kc=P(16), ks=P(16), vc=P(16), vs=P(16), stream=None)
    assert _call(lib.uattn_kv_write_mx, d, kw) == code


@pytest.mark.parametrize("kw,code", SHARED + TOKENS + [(dict(v=P(16)), 1)])
def test_read(lib, kw, code):
    d = dict(kc=P(16), ks=P(16), vc=P(16), vs=P(16), kb=8, vb=4, bt=P(16), seq=P(16), pos=P(16), N=4, B=2, maxp=4, page=16, np=8,
             hkv=2, d=64, k=P(16), v=P(32), st=128, stream=None)
    assert _call(lib.uattn_kv_read_mx, d, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), 1), (dict(hkv=0), 1), (dict(d=32), 2), (dict(kb=6), 2), (dict(vb=-8), 2), (dict(st=127), 1), (dict(st=130), 1),
    (dict(os=127), 1), (dict(os=130), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(ko=None), 1), (dict(vo=None), 1),
    (dict(k=P(24)), 1), (dict(v=P(24)), 1), (dict(ko=P(24)), 1), (dict(vo=P(24)), 1), (dict(N=0), 0), (dict(N=0, k=None, ko=None), 0),
    (dict(hkv=65536, st=1 << 23, os=1 << 23), 2),
    # in place with another stride, and outputs that are each other or the other input
    (dict(ko=P(16), os=256), 1), (dict(vo=P(32), os=256), 1), (dict(ko=P(32)), 1), (dict(vo=P(16)), 1), (dict(vo=P(48)), 1),
])
def test_round(lib, kw, code):
    d = dict(k=P(16), v=P(32), st=128, N=4, hkv=2, d=64, kb=8, vb=4, ko=P(48), vo=P(64), os=128, stream=None)
    assert _call(lib.uattn_kv_round_mx, d, kw) == code


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(hq=3), 1), (dict(hq=66), 2), (dict(scale=0.0), 1), (dict(scale=NAN), 1), (dict(scale=INF), 1), (dict(scale=-1.0), 1),
    (dict(most=-1), 1), (dict(most=0), 1), (dict(most=65), 1), (dict(most=(1 << 24) + 1, maxp=1 << 21), 2), (dict(np=0), 1),
    (dict(q=None), 1), (dict(q=P(24)), 1), (dict(out=None), 1), (dict(out=P(24)), 1), (dict(sl=None), 1),
    (dict(most=2049, maxp=256, ws=None), 3), (dict(most=2049, maxp=256, wsb=1000), 3), (dict(most=2049, maxp=256, ws=P(24)), 3),
    (dict(most=257, maxp=32, hq=34, d=128, ws=None), 3),
    (dict(B=0), 0), (dict(B=0, q=None, kc=None), 0), (dict(B=65536), 2),
])
def test_decode(lib, kw, code):
    d = dict(q=P(16), kc=P(16), ks=P(16), vc=P(16), vs=P(16), kb=8, vb=4, bt=P(16), sl=P(16), B=2, maxp=4, page=16, np=8, most=64,
             hq=4, hkv=2, d=64, scale=0.125, out=P(16), lse=None, ws=P(16), wsb=1 << 24, stream=None)
    assert _call(lib.uattn_decode_mx, d, kw) == code


def test_decode_workspace(lib):
    """Nothing up to 2048 keys where a workgroup folds them; the bf16 decode's partials, without its counters, beyond."""
    need, whole = lib.uattn_decode_mx_workspace_bytes, lib.uattn_decode_workspace_bytes
    assert need(4, 2048, 32, 8, 128) == need(4, 2048, 34, 2, 64) == need(4, 256, 34, 2, 128) == need(4, 1, 1, 1, 64) == 0
    for sizes in ((4, 2049, 32, 8, 128), (4, 257, 34, 2, 128), (300, 100000, 8, 8, 64)):
        b, n, hq, _, d = sizes
        assert need(*sizes) == whole(b, n, hq, d) - (4 * b * hq + 255) // 256 * 256
    for bad in ((0, 4096, 8, 8, 64), (2, -1, 8, 8, 64), (2, 4096, 8, 3, 64), (2, 4096, 8, 0, 64)):
        assert need(*bad) == 0
