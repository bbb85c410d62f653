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
