"""A call's stream belongs to the device that its tensors are on: refused on the host before anything is enqueued."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2505_06653_amd import binding


@pytest.mark.parametrize("device", [1, 7])
def test_a_stream_of_another_device_is_refused(monkeypatch, device):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_check", lambda *a, **k: pytest.fail("enqueued"))
    s = SimpleNamespace(device_index=device, cuda_stream=0x1234)
    x, cb = torch.zeros((1, 64), dtype=torch.bfloat16), np.linspace(-1, 1, 16)
    logits = torch.zeros((1, 9))
    for call in (lambda: binding.bof4_gemv_linear(x, x, 1, 64, 64, cb, x, stream=s), lambda: binding.bof4_gemm_linear(x, 1, 64, cb, x, stream=s),
                 lambda: binding.bof4_gemm_linear_backward(x, 64, 64, cb, x, stream=s), lambda: binding.bof4_token_logprobs(logits, stream=s),
                 lambda: binding.bof4_token_logprobs_backward(logits, logits, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call()
