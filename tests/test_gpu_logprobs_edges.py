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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("h", [3.4e38, -3.4e38, 1e36, 1e30])
def test_gradients_of_the_entropy_up_to_the_largest_number(dtype, out, h):
    """d = -h p (log p + H): p is small where log p is large, so what is finite by the formula has to come out so, and 0 where
    there is no probability."""
    x = torch.full((2, 2003), -math.inf, device=DEV)
    x[:, ::5] = torch.linspace(-80, -20, 401, device=DEV)
    x[:, 7], x[:, 9], x[0, 11], x[:, 12] = 0.0, -1e30, -1.5, torch.finfo(dtype).min
    x = x.to(dtype)
    _, H, _, _, stats = binding.bof4_token_logprobs(x)
    hs, g, t = torch.full((2,), h, device=DEV), torch.ones(2, device=DEV), torch.full((2,), 7, device=DEV)
    for args in ((None, None), (t, g)):
        d = binding.bof4_token_logprobs_backward(x, stats, *args, H, hs, out_dtype=out)
        lp = torch.log_softmax(x.double(), -1)
        p = lp.exp()
        safe = torch.where(p > 0, lp, 0.0)
        want = -float(hs[0]) * p * (safe + H.double()[:, None])
        # lp, of up to 80, and H are off by 2^-24 of 80 each, and so is p: 2^-15 of what is summed up, generously (and of 1: S, a
        # little above 1, is off by 2^-24 at least, and with it log S, however small it is); p below 2^-126 may be 0
        tol = abs(float(hs[0])) * (p * (safe.abs() + H.double()[:, None] + 1) * 2.0 ** -15 + p.clamp(max=2.0 ** -126) * 200) + 2.0
        tol = tol + (want.abs() * 2.0 ** -8 if out == torch.bfloat16 else 0.0)
        assert bool(d.isfinite().all()) and bool(((d.double() - want).abs() <= tol).all())
        assert bool((d[:, 1] == 0).all()) and bool((d[:, 9] == 0).all()) and bool((d[:, 12] == 0).all())
