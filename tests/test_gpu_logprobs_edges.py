"""Token log probabilities and their gradient at the ends of the numbers: rows that are not finite, gradients of the entropy up to
the largest number."""
import math

import pytest
import torch

from paper_2505_06653_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab", [(6, 5), (6, 3001), (600, 5003), (1030, 9001)])
@pytest.mark.parametrize("top", [0, 1, 4])
def test_every_value_of_a_row_with_a_nan_or_inf_is_nan(dtype, n, vocab, top):
    x = torch.randn((n, vocab), generator=torch.Generator(device=DEV).manual_seed(n + vocab), device=DEV).to(dtype)
    x[0, vocab - 1] = math.nan
    x[2, 0] = math.inf
    x[3] = -math.inf
    x[3, vocab // 2] = math.nan
    x[4, 1:] = math.nan
    x[5] = -math.inf  # (no logit at all: not one of them)
    bad, good = [0, 2, 3, 4], [r for r in range(n) if r not in (0, 2, 3, 4)]
    t = torch.ones(n, dtype=torch.int64, device=DEV)
    lp, h, ids, top_lp, stats = binding.bof4_token_logprobs(x, t, top=top)
    for r in (lp, h, stats) + ((top_lp,) if top else ()):
        assert bool(r[bad].isnan().all()) and not bool(r[good].isnan().any())
    assert not top or bool((ids[bad] == -1).all())
    g = torch.ones(n, device=DEV)
    d = binding.bof4_token_logprobs_backward(x, stats, t, g, h, g)
    assert bool(d[bad].isnan().all()) and bool(d[good].isfinite().all())
