"""What the row-wise operators' calls share on the GPU: the stream a call names, and how debug validation reads device data."""
import numpy as np
import pytest

from paper_2609_35140_amd import inputs

pytestmark = pytest.mark.gpu
gu = pytest.importorskip("gpu_util")


@pytest.fixture(scope="module")
def ua():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35140_amd import uattn
    uattn.lib()
    return uattn


def test_handle_of_the_default_stream(ua):
    """stream=0 from inside another stream's context: the call is ordered behind the default stream's work."""
    import torch
    dev, default = torch.cuda.current_device(), torch.cuda.default_stream()
    assert default.cuda_stream == 0
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for handle in (0, 1, default.cuda_stream):
            with ua._elsewhere(dev, handle):
                assert torch.cuda.current_stream() == default
    residual = gu.dev(inputs.normal_bf16((64, 512), 1.0, 361))
    w = gu.dev(np.full(512, 0x3F80, dtype=np.uint16))
    want = ua.residual_norm(residual * 2, w)[1]
    table, ids = residual.clone(), gu.dev_i32(np.arange(64))
    late, a = torch.zeros_like(residual), torch.ones((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(8):          # some milliseconds of the default stream's time, then the inputs
        a = a @ a * 2.0 ** -12
    late.copy_(residual * 2)
    table.copy_(late)
    with torch.cuda.stream(side):
        got = ua.residual_norm(late, w, stream=0)[1]
        rows = ua.embedding(ids, table, stream=default.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(rows, residual * 2)


def _after_a_while(make):
    """On a new stream, some milliseconds of other work and then make()'s copies; nothing waits for it."""
    import torch
    side = torch.cuda.Stream()
    a = torch.ones((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            a = a @ a * 2.0 ** -12
        make()
    return side


def test_validation_reads_what_the_stream_leaves(ua, monkeypatch):
    """UATTN_VALIDATE's copies come behind the work of the call's stream: values that it still has to write are the ones checked."""
    import torch
    V, page = 64, 16
    table = torch.ones((V, 64), dtype=torch.bfloat16, device="cuda")
    z = torch.zeros((3, V), dtype=torch.bfloat16, device="cuda")
    pen, one = torch.ones((3, 3), device="cuda"), torch.ones(3, device="cuda")
    tok = gu.dev_i32([1, 2, 3])
    qkv = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    pages = [torch.zeros((4, 1, page, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    words = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    calls = {  # the array that is checked: values that pass, values that do not, the call
        "ids": ([1, 2, V - 1], [1, 2, V], lambda t, st: ua.embedding(t, table, stream=st)),
        "ids back": ([1, -2, V - 1], [1, 2, V], lambda t, st: ua.embedding_backward(table[:3], t, V, stream=st)),
        "history": ([[0, 1, 2]] * 3, [[0, 1, 4]] * 3, lambda t, st: ua.logits_process(z, tok, t, pen, stream=st)),
        "history back": ([[0, 1, 2]] * 3, [[0, 2, 1]] * 3, lambda t, st: ua.logits_process_backward(z, z, tok, t, pen, stream=st)),
        "mask_rows": ([0, -1, 2], [0, 1, 3], lambda t, st: ua.logits_process(z, mask=words, mask_rows=t, stream=st)),
        "targets back": ([0, 1, 2], [0, 1, V], lambda t, st: ua.logprob_backward(z, t, one, stream=st)),
        "targets": ([0, 1, 2], [0, -1, 2], lambda t, st: ua.logprob(z, t, stream=st)),
        "offsets": ([0, 1, 3], [0, 1, 4], lambda t, st: ua.prefill(qkv, qkv, qkv, t, 2, stream=st)),
        "lengths": ([1, 17, 32], [1, 17, 33],
                    lambda t, st: ua.decode(qkv, *pages, gu.dev_i32([[0, 1], [2, 3], [1, 2]]), t, 32, stream=st)),
        "positions": ([0, 17, -1], [0, 17, 32],
                      lambda t, st: ua.kv_write(qkv, qkv, gu.dev_i32([[0, 1], [2, 3]]), gu.dev_i32([0, 1, 1]), t, *pages, stream=st)),
    }
    for name, (good, bad, call) in calls.items():
        call(gu.dev_i32(good), None)
    torch.cuda.synchronize()
    monkeypatch.setenv("UATTN_VALIDATE", "1")
    for name, (good, bad, call) in calls.items():
        print(name, flush=True)
        for first, last in ((bad, good), (good, bad)):
            t, end = gu.dev_i32(first), gu.dev_i32(last)
            side = _after_a_while(lambda: t.copy_(end))
            if last is good:
                call(t, side)
            else:
                with pytest.raises(ua.UattnError, match="EINVAL"):
                    call(t, side)
            torch.cuda.synchronize()
    # a gradient of 0 lets any target pass: the weights too are read behind the stream's work
    tg, dl = gu.dev_i32([0, 1, V]), torch.ones(3, device="cuda")
    side = _after_a_while(lambda: dl[2:].zero_())
    assert not ua.logprob_backward(z, tg, dl, stream=side)[2].any()
    torch.cuda.synchronize()


def test_validation_refuses_a_captured_call(ua, monkeypatch):
    """Nothing runs while a stream is captured, so its values cannot be checked: the call is refused, the capture goes on, and
    without validation the same call is captured."""
    import torch
    ids = gu.dev_i32([0, 3, 1])
    table = gu.dev(inputs.normal_bf16((4, 64), 1.0, 362))
    ua.embedding(ids, table)
    marks = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        marks.add_(1.0)
        monkeypatch.setenv("UATTN_VALIDATE", "1")
        with pytest.raises(ua.UattnError, match="EINVAL"):
            ua.embedding(ids, table)
        monkeypatch.delenv("UATTN_VALIDATE")
        rows = ua.embedding(ids, table)
    for n in (1, 2, 3):
        graph.replay()
        torch.cuda.synchronize()
        assert bool((marks == n).all()) and torch.equal(rows, table[ids.long()])


def test_logprob_backward_in_place_is_refused(ua):
    import torch
    z = gu.dev(inputs.normal_bf16((3, 64), 1.0, 363))
    was = z.clone()
    with pytest.raises(ua.UattnError, match="EINVAL"):
        ua.logprob_backward(z, gu.dev_i32([1, 2, 3]), torch.ones(3, device="cuda"), out=z)
    assert torch.equal(z, was)
