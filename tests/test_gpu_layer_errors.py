"""A launch that CUDA refuses is reported by the call that it belongs to, and by no call after it."""
import ctypes

import pytest
import torch

from test_gpu_experts import make

pytestmark = pytest.mark.gpu

binding = pytest.importorskip("paper_2609_36301_b200.binding")


@pytest.mark.parametrize("op", ["pairs", "tiles", "backward", "combine", "combine_ring", "combine_backward", "dispatch"])
def test_a_refused_launch_is_reported_once(op):
    """Every launch into a capture that has become invalid is refused on the host.  The same call on another stream is right after it."""
    T, h, s, M, k = (1300, 1024, 16, 8, 2) if op == "combine_ring" else (64, 64, 16, 8, 2)
    X, W1, W2, idx, offsets, pairs, gate, dout = make(T, h, s, M, k)
    y, hidden = torch.zeros((T * k, h), device="cuda").bfloat16(), torch.zeros((T * k, 2 * s), device="cuda").bfloat16()
    w = [torch.ones(h, device="cuda") for _ in range(3)]
    ws = torch.empty(binding.experts_workspace(T, h, s, M, k, True) + binding.combine_workspace(T, h), device="cuda", dtype=torch.uint8)
    counts = (offsets[1:] - offsets[:-1]).contiguous()
    rows = [torch.empty_like(X) for _ in range(2)]
    grads = [torch.empty_like(v) for v in (X, gate, W1, W2)]
    cols = [torch.empty_like(v) for v in w]

    def call(stream):
        if op == "pairs":
            binding.more_experts(X, W1, W2, idx, None, None, y, path=binding.EXPERTS_PAIRS, stream=stream)
        elif op == "tiles":
            binding.more_experts(X, W1, W2, idx, offsets, pairs, y, hidden, workspace=ws, stream=stream)
        elif op == "backward":
            binding.more_experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, *grads, workspace=ws, stream=stream)
        elif op == "dispatch":
            binding.more_dispatch(idx, counts, offsets, pairs, stream=stream)
        elif op == "combine_backward":
            binding.more_combine_backward(X, dout, dout, X, *w, 1e-6, *rows, *cols, workspace=ws, stream=stream)
        else:
            binding.more_combine(y, gate, X, *w, 1e-6, *rows, stream=stream)

    other = torch.cuda.Stream()
    call(other)
    torch.cuda.synchronize()
    runtime, stream = ctypes.CDLL("libcudart.so.12"), torch.cuda.Stream()          # (the one that torch has loaded; its graphs stay out of it)
    handle, graph = ctypes.c_void_p(stream.cuda_stream), ctypes.c_void_p()
    assert runtime.cudaStreamBeginCapture(handle, 1) == 0                          # (of this thread)
    try:
        assert runtime.cudaStreamSynchronize(handle) != 0                          # not allowed in a capture, which it makes invalid
        with pytest.raises(binding.MoreRouteError):
            call(stream)
        call(other)                                                                # nothing of it is left
    finally:
        assert runtime.cudaStreamEndCapture(handle, ctypes.byref(graph)) != 0
        runtime.cudaGetLastError()
    call(other)
    torch.cuda.synchronize()
    assert float(torch.rand(8, device="cuda").sum()) > 0
