"""Calls without a stream argument run on torch's current stream: the handle the binding takes is the current one's."""
import pytest

from conftest import gpu_available

pytestmark = pytest.mark.gpu


def test_current_stream_handle():
    if not gpu_available():
        pytest.skip("no GPU")
    import threading

    import torch
    from paper_2608_15602_amd import fluxbin as fb
    assert fb._stream(None) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert fb._stream(None) == side.cuda_stream
        other = []
        t = threading.Thread(target=lambda: other.append((fb._stream(None), torch.cuda.current_stream().cuda_stream)))
        t.start()
        t.join()
        assert other[0][0] == other[0][1]   # the current stream is a thread's own
    assert fb._stream(None) == torch.cuda.current_stream().cuda_stream
    assert fb._stream(side) == side.cuda_stream and fb._stream(side.cuda_stream) == side.cuda_stream


def test_fill_before_the_other_stream_waits():
    """An output filled on the current stream, then attention on another stream that has waited for it: the attention's values
    stay, also on streams that nothing has used before."""
    if not gpu_available():
        pytest.skip("no GPU")
    import numpy as np
    import torch
    from paper_2608_15602_amd import fluxbin as fb
    from test_gpu_kv8 import Setup
    s = Setup(fb, 2, 2, 128, 64, 300, seed=18)
    s.append([300, 7])
    q = s.dev(s.rng.standard_normal((2, 16, 128)).astype(np.float16))
    a = s.arrays([0, 1, 2], s.length)
    ref = fb.fluxbin_kv8_attention(s.cache, q, *a)
    for _ in range(8):
        side = torch.cuda.Stream()
        out, ws = torch.zeros_like(ref), fb.make_kv8_workspace(s.cache, 2, 2, 16)
        side.wait_stream(torch.cuda.current_stream())
        fb.fluxbin_kv8_attention(s.cache, q, *a, out=out, workspace=ws, stream=side)
        side.synchronize()
        assert torch.equal(out, ref)
