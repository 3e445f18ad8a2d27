"""What the products and layers take for x: [n_tokens, cols] or one token's [cols], refused on the host otherwise."""
import numpy as np
import pytest
import torch

from paper_2505_06653_amd import binding

BF16 = torch.bfloat16


@pytest.mark.parametrize("shape", [(), (64, 2, 2), (1, 64, 2), (2, 1, 64), (64, 1), (63,), (3, 65), (1, 64, 64)])
def test_other_shapes_are_refused(monkeypatch, shape):
    """(A tensor of three dimensions whose first is as wide as the matrix passed for one token.)"""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # what tensors of the host say
    monkeypatch.setattr(binding, "_check", lambda *a, **k: pytest.fail("enqueued"))
    monkeypatch.setattr(binding, "_stream", lambda stream: None)
    x, cb = torch.zeros(shape, dtype=BF16), np.linspace(-1, 1, 16)
    codes, scales = torch.zeros(64, dtype=torch.uint8), torch.zeros(8, dtype=torch.float16)
    packed = torch.zeros(binding.bof4_gemm_packed_bytes(2, 64), dtype=torch.uint8)
    for call in (lambda: binding.bof4_gemv(codes, scales, 2, 64, 32, cb, x), lambda: binding.bof4_gemm(packed, 2, 64, cb, x),
                 lambda: binding.bof4_gemv_linear(codes, scales, 2, 64, 32, cb, x), lambda: binding.bof4_gemm_linear(packed, 2, 64, cb, x)):
        with pytest.raises(ValueError, match="n_tokens, cols"):
            call()


def test_one_token_and_several_are_taken():
    for shape in ((64,), (1, 64), (5, 64)):
        assert binding._tokens(torch.zeros(shape, dtype=BF16), 64).shape == (shape[0] if len(shape) == 2 else 1, 64)
