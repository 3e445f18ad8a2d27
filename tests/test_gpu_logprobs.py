"""Token log probabilities, entropy, alternatives and their gradient against the definitions in binary64.

Bounds.  One step: U = 2^-24.  u = x - m is off by |u| U, its exponential by 2 |u| U and the instruction's 2 U; in the mean over
p that is a few U times the entropy-like sum E = sum p |u| <= log(vocab).  A sum is a chain of at most vocab / 64 additions in
a lane (three roundings each where the maximum moves) and 32 more: with C = 128 + vocab / 16 + 4 E, log S is off by C U, a log
probability by (C + 4 |lp|) U, and the entropy, with T / S <= E, by (C + 2 E C) U."""
import math

import numpy as np
import pytest
import torch

from paper_2505_06653_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def reference(logits, target):
    """log p, p, entropy, E and log probabilities of the targets in binary64 (rows of ordinary numbers and -inf)."""
    x = logits.double()
    m = x.amax(1, keepdim=True)
    u = torch.where(x == -math.inf, -math.inf, x - m)
    logp = u - u.exp().sum(1, keepdim=True).log()
    p = logp.exp()
    safe = torch.where(p > 0, logp, 0.0)
    lp = None
    if target is not None:
        ok = (target >= 0) & (target < x.shape[1])
        lp = torch.where(ok, logp.gather(1, torch.where(ok, target, 0)[:, None])[:, 0], 0.0)
    return logp, p, -(p * safe).sum(1), (p * torch.where(p > 0, -u, 0.0)).sum(1), lp


def bounds(logits, E, lp):
    c = 128 + logits.shape[1] / 16 + 4 * E
    return (c + 4 * (lp.abs() if lp is not None else 0.0)) * U, (c + 2 * E * c) * U


def check(logits, target=None, top=0, **kw):
    logp, p, entropy, E, lp = reference(logits, target)
    g_lp, g_h, ids, top_lp, stats = binding.bof4_token_logprobs(logits, target, top=top, **kw)
    b_lp, b_h = bounds(logits, E, lp)
    if target is not None:
        same = (g_lp.double() == lp)  # (-inf among them)
        assert bool((same | ((g_lp.double() - lp).abs() <= b_lp)).all())
    assert bool(((g_h.double() - entropy).abs() <= b_h).all()), float((g_h.double() - entropy).abs().max())
    assert torch.equal(stats[:, 0].double(), logits.double().amax(1))
    if top:
        n_alt = (logits > -math.inf).sum(1)
        order = torch.sort(logits.float(), dim=1, descending=True, stable=True).indices[:, :top]
        k = order.shape[1]
        place = torch.arange(top, device=DEV)[None, :] < n_alt[:, None]
        want = torch.full((logits.shape[0], top), -1, dtype=torch.int64, device=DEV)
        want[:, :k] = order
        want = torch.where(place, want, -1)
        assert torch.equal(ids, want)
        w_lp = torch.where(place, logp.gather(1, want.clamp(min=0)), -math.inf)
        diff = torch.where(place, (top_lp.double() - w_lp).abs(), 0.0)
        c = (128 + logits.shape[1] / 16 + 4 * E)[:, None]
        assert bool((diff <= (c + 4 * torch.where(place, w_lp, 0.0).abs()) * U).all())
        assert bool((torch.where(place, 0.0, top_lp) == torch.where(place, 0.0, -math.inf)).all())
    return g_lp, g_h, ids, top_lp, stats


def make(n, vocab, dtype, seed, spread=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = spread * torch.randn((n, vocab), generator=g, device=DEV)
    x[:, (7 * seed) % vocab] += 9.0
    t = torch.randint(-1, vocab, (n,), generator=g, device=DEV)
    return x.to(dtype), t


SHAPES = [(1, 1), (2, 2), (1, 5), (3, 63), (3, 64), (5, 65), (2, 1000), (300, 2049), (7, 50257), (3, 128000), (1, 300001),
          (1000, 1023), (2, 4096), (2, 4097), (515, 8193), (1030, 2047), (1025, 100003)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab", SHAPES)
@pytest.mark.parametrize("top", [0, 1, 20, 64])
def test_against_binary64(n, vocab, dtype, top):
    x, t = make(n, vocab, dtype, n + vocab)
    check(x, t, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seed", range(6))
def test_random_shapes(seed, dtype):
    rng = np.random.default_rng(seed)
    n, vocab = int(np.exp(rng.uniform(0, np.log(600)))), int(np.exp(rng.uniform(0, np.log(60000))))
    x, t = make(n, vocab, dtype, seed, spread=float(rng.uniform(0.1, 30)))
    check(x, t, int(rng.integers(0, 65)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first,extra", [(1, 0), (3, 5), (0, 1), (8, 8)])
def test_rows_of_any_stride_and_alignment(dtype, first, extra):
    whole, t = make(9, 5003 + first + extra, dtype, 3)
    view = whole[:, first:first + 5003]
    t = t.clamp(max=5002)
    a = check(view, t, 7)
    b = binding.bof4_token_logprobs(view.contiguous(), t, top=7)
    for p, q in zip(a, b):  # ids equal; sums within their bounds, whatever the rows' alignment
        assert torch.equal(p, q) if p.dtype == torch.int64 else torch.allclose(p, q, rtol=0, atol=1e-4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks(dtype):
    n, vocab = 12, 3001
    x, _ = make(n, vocab, dtype, 5)
    t = torch.arange(n, device=DEV) * 17
    mask = torch.rand((n, vocab), device=DEV) < 0.5
    mask[0] = True
    mask[0, 5] = False          # one token left
    mask[1] = True
    mask[1, 3000] = False       # the last one
    mask[2] = True
    mask[2, :3] = False
    check(x.masked_fill(mask, -math.inf), t, 20)
    low = torch.finfo(dtype).min  # the type's lowest value in masked places
    y = x.masked_fill(mask, low)
    check(y, t, 2)
    check(torch.full_like(x, low), t, 5)   # a row masked that way is uniform
    check(torch.full_like(x, torch.finfo(dtype).max), t, 5)


def test_rows_without_any_logit_and_rows_that_are_not_finite():
    n, vocab = 9, 5000
    x, t = make(n, vocab, torch.float32, 8)
    t = torch.full_like(t, 3)
    x[1] = -math.inf
    x[3, 4999] = math.nan
    x[4, 3] = math.inf
    x[5] = math.nan
    x[6, 17] = math.inf
    x[6, 18] = -math.inf
    lp, h, ids, top, stats = binding.bof4_token_logprobs(x, t, top=4)
    assert lp[1] == -math.inf and h[1] == 0 and ids[1].tolist() == [-1] * 4 and top[1].tolist() == [-math.inf] * 4
    assert stats[1].tolist() == [-math.inf, 0.0]
    for r in (3, 4, 5, 6):
        assert torch.isnan(lp[r]) and torch.isnan(h[r]) and torch.isnan(top[r]).all() and ids[r].tolist() == [-1] * 4
    keep = [0, 2, 7, 8]
    check(x[keep].contiguous(), t[keep], 4)
    g = torch.ones(n, device=DEV)
    d = binding.bof4_token_logprobs_backward(x, stats, t, g, h, g)
    assert (d[1] == 0).all()
    for r in (3, 4, 5, 6):
        assert torch.isnan(d[r]).all()
    assert torch.isfinite(d[keep]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 300])
def test_ties_and_orders(dtype, n):
    vocab = 9001
    check(torch.zeros((n, vocab), dtype=dtype, device=DEV), None, 64)
    up = torch.linspace(-20, 20, vocab, device=DEV).to(dtype).repeat(n, 1)
    check(up, None, 64)
    check(up.flip(1).contiguous(), None, 64)
    zeros = torch.zeros((n, vocab), dtype=dtype, device=DEV)
    zeros[:, ::2] = -0.0   # equal to +0
    check(zeros, None, 33)
    few = (torch.arange(vocab, device=DEV) % 3).to(dtype).repeat(n, 1)
    check(few, None, 50)
    late = zeros.clone()
    late[:, -64:] = 1.0    # all alternatives at the very end
    check(late, None, 64)
    check(torch.full((n, 3), 2.0, dtype=dtype, device=DEV), None, 64)


def test_one_token_takes_all_and_wide_ranges():
    x = torch.zeros((3, 2000), device=DEV)
    x[:, 7] = 60.0
    x[1, 7] = 1e30
    x[2] = -1e30
    x[2, 9] = 3e38
    check(x, torch.tensor([7, 7, 9], device=DEV), 3)
    check(x, torch.tensor([8, 8, 8], device=DEV), 3)


def test_targets_outside_the_vocabulary_ask_for_nothing():
    x, _ = make(5, 777, torch.float32, 1)
    t = torch.tensor([-100, -1, 777, 1 << 40, 776], device=DEV)
    lp = check(x, t)[0]
    assert lp[:4].tolist() == [0, 0, 0, 0] and lp[4] < 0
    g = torch.ones(5, device=DEV)
    _, h, _, _, stats = binding.bof4_token_logprobs(x)
    d = binding.bof4_token_logprobs_backward(x, stats, t, g)
    assert (d[:4] == 0).all() and (d[4] != 0).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab", [(1, 1), (2, 7), (3, 1001), (40, 32000), (2, 50257), (300, 64)])
@pytest.mark.parametrize("which", ["logprob", "entropy", "both"])
def test_gradient_against_the_formula(n, vocab, dtype, out, which):
    x, t = make(n, vocab, dtype, 11)
    if vocab > 100:
        x[:, 3::5] = -math.inf
        t = torch.where(t % 5 == 3, t - 1, t)
    gen = torch.Generator(device=DEV).manual_seed(2)
    g, h = torch.randn(n, generator=gen, device=DEV), torch.randn(n, generator=gen, device=DEV)
    logp, p, H, E, lp = reference(x, t)
    _, entropy, _, _, stats = binding.bof4_token_logprobs(x)
    has = (t >= 0)
    want = torch.zeros_like(logp)
    size = torch.zeros_like(logp)  # what the roundings are relative to
    safe = torch.where(p > 0, logp, 0.0)
    args = {}
    if which != "entropy":
        gg = torch.where(has, g, 0.0).double()[:, None]
        want -= gg * p
        size += gg.abs() * p
        want.scatter_add_(1, t.clamp(min=0)[:, None], gg)
        args.update(targets=t, d_logprob=g)
    if which != "logprob":
        hh = h.double()[:, None]
        want -= hh * p * (safe + H[:, None])
        size += hh.abs() * p * (safe.abs() + H[:, None] + 1)
        args.update(entropy=entropy, d_entropy=h)
    d = binding.bof4_token_logprobs_backward(x, stats, out_dtype=out, **args)
    # log p is off by (C + 4 |log p|) U, p by that relatively, the entropy by (C + 2 E C) U, and four more roundings
    c = (128 + vocab / 16 + 4 * E)[:, None]
    rel = (2 * c + 2 * E[:, None] * c + 8 * safe.abs() + 8) * U
    tol = size * rel + (want.abs() * 2.0 ** -8 + 2.0 ** -133 if out == torch.bfloat16 else want.abs() * 2 * U) + 2.0 ** -126
    assert d.dtype == out and bool(((d.double() - want).abs() <= tol).all())
    if vocab > 100:
        assert (d[:, 3::5] == 0).all()


def test_gradient_against_differences():
    """Central differences of the binary64 definition: their own error is h^2 / 6 times third derivatives of order one, and
    the log probability's rounding over h."""
    x, t = make(2, 9, torch.float32, 4, spread=1.0)
    t = torch.tensor([2, 5], device=DEV)
    g, h = torch.tensor([0.7, -1.3], device=DEV), torch.tensor([0.4, 0.9], device=DEV)
    _, entropy, _, _, stats = binding.bof4_token_logprobs(x, t)
    d = binding.bof4_token_logprobs_backward(x, stats, t, g, entropy, h)

    def loss(y):
        _, _, H, _, lp = reference(y, t)
        return (lp * g.double() + H * h.double()).sum()

    step = 1e-4
    for i in range(2):
        for j in range(9):
            e = torch.zeros((2, 9), dtype=torch.float64, device=DEV)
            e[i, j] = step
            diff = (loss(x.double() + e) - loss(x.double() - e)) / (2 * step)
            assert abs(float(d[i, j]) - float(diff)) < 1e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_in_place_into_strided_rows_and_nothing_else(dtype):
    n, vocab = 6, 1003
    x, t = make(n, vocab, dtype, 6)
    g = torch.linspace(-1, 1, n, device=DEV)
    _, _, _, _, stats = binding.bof4_token_logprobs(x, t)
    want = binding.bof4_token_logprobs_backward(x, stats, t, g)
    wide = torch.full((n, vocab + 10), 7.0, dtype=dtype, device=DEV)
    view = wide[:, 3:3 + vocab]
    binding.bof4_token_logprobs_backward(x, stats, t, g, out=view)
    assert torch.equal(view, want) and (wide[:, :3] == 7).all() and (wide[:, 3 + vocab:] == 7).all()
    wide[:, 3:3 + vocab] = x
    binding.bof4_token_logprobs_backward(view, stats, t, g, out=view)
    assert torch.equal(view, want) and (wide[:, :3] == 7).all() and (wide[:, 3 + vocab:] == 7).all()


@pytest.mark.parametrize("n,vocab", [(2, 100003), (700, 3001), (1100, 2001)])
def test_equal_bits_on_every_call_other_streams_and_captured(n, vocab):
    x, t = make(n, vocab, torch.float32, 9)
    g = torch.ones(n, device=DEV)
    first = binding.bof4_token_logprobs(x, t, top=9)
    d_first = binding.bof4_token_logprobs_backward(x, first[4], t, g, first[1], g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    second = binding.bof4_token_logprobs(x, t, top=9, stream=s)
    s.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    ws = torch.empty(binding.bof4_token_logprobs_workspace_bytes(n, vocab, 9), dtype=torch.uint8, device=DEV)
    ws.fill_(0xff)
    graph = torch.cuda.CUDAGraph()
    xs = x.clone()
    with torch.cuda.graph(graph):
        out = binding.bof4_token_logprobs(xs, t, top=9, ws=ws)
        d = binding.bof4_token_logprobs_backward(xs, out[4], t, g, out[1], g)
    for k in range(3):
        y = torch.roll(x, k, 1)
        xs.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        want = binding.bof4_token_logprobs(y, t, top=9)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        assert torch.equal(d, binding.bof4_token_logprobs_backward(y, want[4], t, g, want[1], g))
    assert torch.equal(d_first, binding.bof4_token_logprobs_backward(x, first[4], t, g, first[1], g))


def test_offsets_past_32_bits():
    """Rows that begin beyond 2^32 bytes and 2^31 elements of the first."""
    vocab, ld = 1000, (1 << 31) + 8
    whole = torch.empty(ld + vocab + 64, dtype=torch.bfloat16, device=DEV)
    x, t = make(2, vocab, torch.bfloat16, 12)
    view = whole[:ld + vocab].as_strided((2, vocab), (ld, 1))
    view.copy_(x)
    check(view, t.clamp(min=0), 5)
    _, _, _, _, stats = binding.bof4_token_logprobs(x, t)
    g = torch.ones(2, device=DEV)
    want = binding.bof4_token_logprobs_backward(x, stats, t, g)
    got = binding.bof4_token_logprobs_backward(view, stats, t, g, out=view)
    assert torch.equal(got, want)


def test_refusals():
    x, t = make(4, 100, torch.float32, 1)
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs(x.half(), t)
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs(x.t(), t)
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs(x, t[:3])
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs(x, t.int())
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs(x.cpu(), t)
    with pytest.raises(binding.Bof4Error):
        binding.bof4_token_logprobs(x, t, top=65)
    with pytest.raises(binding.Bof4Error):
        binding.bof4_token_logprobs(x, t, ws=torch.empty(0, dtype=torch.uint8, device=DEV))
    _, h, _, _, stats = binding.bof4_token_logprobs(x, t)
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs_backward(x, stats, t)
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs_backward(x, stats, entropy=h)
    with pytest.raises(ValueError):
        binding.bof4_token_logprobs_backward(x, stats[:2], t, h)


def test_results_changed_in_place_leave_what_the_gradient_needs():
    """Inside an autograd function: the caller masks the log probabilities in place, the statistics stay as they were saved."""
    class LogProb(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, t):
            logprob, entropy, _, top, stats = binding.bof4_token_logprobs(x, t, top=3)
            assert not any(r._is_view() for r in (logprob, entropy, top, stats))
            ctx.save_for_backward(x, stats, t, entropy)
            return logprob

        @staticmethod
        def backward(ctx, g):
            x, stats, t, entropy = ctx.saved_tensors
            return binding.bof4_token_logprobs_backward(x, stats, t, g.contiguous()), None

    x = make(6, 1000, torch.float32, 3)[0].requires_grad_(True)
    t = torch.arange(6, device=DEV) * 150
    keep = torch.tensor([1.0, 0.0, 2.0, 1.0, 0.0, 1.0], device=DEV)
    logprob = LogProb.apply(x, t)
    logprob *= keep
    logprob.sum().backward()
    want = keep[:, None].double() * (torch.nn.functional.one_hot(t, 1000) - torch.softmax(x.detach().double(), -1))
    # exp of a difference rounded at 2^-24 of up to 30, and the sum's own error: below 64 half steps of the largest gradient
    assert float((x.grad.double() - want).abs().max()) <= 64 * 2.0 ** -24 * 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_gradients_of_the_entropy_stay_finite_next_to_logits_without_probability(dtype):
    """p = 0 there, and with it the gradient, however large d_entropy is."""
    n, vocab = 5, 3001
    x, t = make(n, vocab, dtype, 4)
    x[:, ::3] = -math.inf
    x[:, 1::7] = -1e30
    t[:] = 2
    _, entropy, _, _, stats = binding.bof4_token_logprobs(x, t)
    g, h = torch.ones(n, device=DEV), torch.tensor([1e9, -1e9, 1e20, 1e30, 1.0], device=DEV)
    d = binding.bof4_token_logprobs_backward(x, stats, t, g, entropy, h, out_dtype=torch.float32).double()
    lp = torch.log_softmax(x.double(), -1)
    p = lp.exp()
    slope = p * (torch.where(p > 0, lp, 0.0) + entropy.double()[:, None])
    want = g[:, None] * (torch.nn.functional.one_hot(t, vocab) - p) - h.double()[:, None] * slope
    # lp, of up to 32, and H are off by some 2^-24 of 32 each, twice over in p: 2^-17 of what is summed up, generously
    size = g[:, None] + h.double().abs()[:, None] * p * (torch.where(p > 0, lp.abs(), 0.0) + entropy.double()[:, None])
    assert bool(((d - want).abs() <= 2.0 ** -17 * size).all())
