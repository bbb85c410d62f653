"""Sizes of 2^31 and more in the Python binding: refused before the library, whose 32-bit arguments would lose their high bits.

Tensors of such shapes stand here without memory ("meta" tensors that say they are on a GPU), and nothing may reach the library.
"""
import pytest
import torch

BF16, I32, F32 = torch.bfloat16, torch.int32, torch.float32
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
            assert name.endswith("workspace_bytes"), f"{name} was reached"
            return lambda *sizes: 16

    monkeypatch.setattr(uattn, "_load", Library)
    monkeypatch.setattr(uattn, "_elsewhere", lambda device, stream: None)
    monkeypatch.setattr(uattn, "_stream_on", lambda device: 0)
    monkeypatch.setattr(uattn, "_stream", lambda stream: 0)
    monkeypatch.setattr(uattn, "new_workspace", lambda nbytes, device: t((nbytes,), torch.uint8))
    for f in (uattn.residual_norm_backward_workspace_bytes, uattn.embedding_backward_workspace_bytes):
        f.cache_clear()
    yield uattn
    for f in (uattn.residual_norm_backward_workspace_bytes, uattn.embedding_backward_workspace_bytes):
        f.cache_clear()


def _norm(T, H):
    return lambda ua: ua.residual_norm(t((T, H)), t((H,)), x=t((T, H)))


def _norm_grad(T, H):
    return lambda ua: ua.residual_norm_backward(t((T, H)), None, t((T, H)), t((H,)))


def _embed(T, V, H):
    return lambda ua: ua.embedding(t((T,), I32), t((V, H)))


def _embed_grad(T, V, H, given=False):
    return lambda ua: ua.embedding_backward(t((T, H)), t((T,), I32), V, grad=t((V, H), F32) if given else None)


def _logits(T=2, V=64, N=5, M=3, K=1):
    parts = dict(tokens=t((N,), I32), history=t((T, 3), I32), penalties=t((T, 3), F32), mask=t((K, (V + 31) // 32), I32),
                 mask_rows=t((T,), I32))
    bias = dict(bias_ids=t((M,), I32), bias_values=t((M,), F32), bias_rows=t((T, 2), I32))
    return parts, bias, t((T, V))


def _process(**kw):
    def f(ua):
        parts, bias, z = _logits(**kw)
        ua.logits_process(z, **parts, **bias)
    return f


def _process_grad(**kw):
    def f(ua):
        parts, _, z = _logits(**kw)
        ua.logits_process_backward(z, z, **parts)
    return f


def _logp_grad(T, V):
    return lambda ua: ua.logprob_backward(t((T, V)), t((T,), I32), t((T,), F32))


ROWS = [_norm(WRAPS, 8), _norm(2 ** 31, 8), _norm(2, WRAPS), _norm_grad(WRAPS, 8), _norm_grad(2, WRAPS), _embed(WRAPS, 9, 8),
        _embed(4, WRAPS, 8), _embed(4, 9, WRAPS), _embed_grad(WRAPS, 9, 8), _embed_grad(4, WRAPS, 8), _embed_grad(4, WRAPS, 8, True),
        _embed_grad(4, 9, WRAPS), _process(T=WRAPS), _process(V=WRAPS), _process(N=2 ** 32 + 5), _process(M=2 ** 32 + 5),
        _process(K=WRAPS), _process_grad(T=WRAPS), _process_grad(V=2 ** 31), _process_grad(N=2 ** 31 + 1), _process_grad(K=2 ** 31),
        _logp_grad(WRAPS, 8), _logp_grad(2, WRAPS)]


def _prefill(T=4, H=2, K=1, D=64, S=1, most=4, back=False):
    def f(ua):
        q, k, cu = t((T, H, D)), t((T, K, D)), t((S + 1,), I32)
        if back:
            return ua.prefill_backward(q, k, k, q, q, t((T, H), F32), cu, most)
        return ua.prefill(q, k, k, cu, most)
    return f


def _decode(B=2, H=2, K=1, D=64, page=16, P=4, maxp=4, most=40, how="decode"):
    def f(ua):
        q, pages, table, lens = t((B, H, D)), t((P, K, page, D)), t((B, maxp), I32), t((B,), I32)
        if how == "steps":
            return ua.DecodeSteps(t((3, B, H, D)), pages, pages, table, t((3, B), I32), most, t((3, B, H, D)))
        return getattr(ua, how)(q, pages, pages, table, lens, most)
    return f


def _kv(N=2, B=2, P=4, maxp=4, K=1, page=16, D=64):
    pages = t((P, K, page, D))
    return lambda ua: ua.kv_write(t((N, K, D)), t((N, K, D)), t((B, maxp), I32), t((N,), I32), t((N,), I32), pages, pages)


def _rope(T=2, H=2, K=1, D=64, P=8):
    return lambda ua: ua.qk_norm_rope(t((T, H, D)), t((T, K, D)), t((T,), I32), t((D,)), t((D,)), t((P, D // 2, 2), F32))


def _head(T=2, V=8, H=64, logp=False):
    if logp:
        return lambda ua: ua.lm_head_logprob(t((T, H)), t((V, H)), t((T,), I32), out=t((T,), F32))
    return lambda ua: ua.lm_head(t((T, H)), t((V, H)), out=t((T, V)))


OTHERS = [_prefill(T=WRAPS), _prefill(H=WRAPS), _prefill(K=WRAPS), _prefill(D=WRAPS), _prefill(S=WRAPS), _prefill(most=WRAPS),
          _prefill(most=-WRAPS), _prefill(T=WRAPS, back=True), _prefill(most=WRAPS, back=True), _decode(B=WRAPS), _decode(P=WRAPS),
          _decode(maxp=WRAPS), _decode(most=WRAPS), _decode(page=2 ** 32 + 16), _decode(P=WRAPS, how="decode_noalloc"),
          _decode(most=WRAPS, how="decode_noalloc"), _decode(P=WRAPS, how="steps"), _decode(most=WRAPS, how="steps"),
          lambda ua: ua.logprob(t((WRAPS, 8)), t((WRAPS,), I32)), lambda ua: ua.logprob(t((2, WRAPS)), t((2,), I32)), _kv(N=WRAPS),
          _kv(B=WRAPS), _kv(P=WRAPS), _kv(maxp=WRAPS), lambda ua: ua.rope_cache(WRAPS, 64, 1e4, out=t((WRAPS, 32, 2), F32)),
          _rope(T=WRAPS), _rope(P=WRAPS), _head(T=WRAPS), _head(V=WRAPS), _head(H=WRAPS), _head(T=WRAPS, logp=True),
          _head(V=WRAPS, logp=True)]


@pytest.mark.parametrize("call", ROWS + OTHERS)
def test_sizes_past_32_bits_are_refused(ua, call):
    with pytest.raises(ValueError, match="2\\^31"):
        call(ua)


def test_ordinary_sizes_reach_the_library(ua):
    for call in (_norm(4, 8), _norm_grad(4, 8), _embed(4, 9, 8), _embed_grad(4, 9, 8), _process(), _process_grad(), _logp_grad(2, 64),
                 _prefill(), _prefill(back=True), _decode(), _decode(how="decode_noalloc"),
                 lambda ua: ua.logprob(t((2, 8)), t((2,), I32)), _kv(), _rope(), _head(), _head(logp=True)):
        with pytest.raises(AssertionError, match="was reached"):
            call(ua)


def test_workspaces_of_invalid_sizes():
    """0, as for other sizes that the call refuses; a workspace of the size without its high bits would be too small."""
    from paper_2609_35140_amd import uattn as ua
    for n in (WRAPS, 2 ** 31, -WRAPS):
        assert ua.residual_norm_backward_workspace_bytes(n, 64) == ua.embedding_backward_workspace_bytes(n, 64) == 0
        assert ua.embedding_backward_workspace_bytes(4, n) == ua.prefill_backward_workspace_bytes(n, 4) == 0
        assert ua.decode_workspace_bytes(2, n, 4, 64) == ua.lm_head_logprob_workspace_bytes(n, 256) == 0
