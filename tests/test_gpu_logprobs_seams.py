"""Every logit counts exactly once, wherever a row is cut: at the ends of rows, of 16-byte words, tiles, waves and parts.

Bounds, U = 2^-24.  A lane adds the 16 (bfloat16: 32) logits of each of its tiles to two sums in turn, so a sum is a chain of 8
(16) roundings a tile and three more where the maximum moves; then two sums, 64 lanes (6 steps), up to four waves and up to 64 parts
(6 steps) join, three roundings each, and an exponential is off by 2 U and 2 |u| U.  With C = (8 or 16 + 3) tiles + 3 (1 + 6 + 4 + 6) + 2
+ 4 E, E = sum p |u|: log S is off by (C + 1) U and two half steps of itself, a log probability by that and 2 |lp| U, the entropy, T / S
at most E, by (C + 1 + 2 E C) U and two half steps of log S and H.  Nothing grows with the vocabulary but the tiles."""
import math

import pytest
import torch

from paper_2505_06653_amd import binding
from test_gpu_logprobs import reference
from test_host_logprobs_plan import plan  # noqa: F401 (a fixture: how rows are cut)

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


def rows_at(n, vocab, dtype, extra=0, first=0):
    """n rows of `vocab` inside wider ones, so that they begin at changing places of 16-byte words."""
    return torch.zeros((n, first + vocab + extra), dtype=dtype, device=DEV)[:, first:first + vocab]


def bounds(plan, x, E, lp, H):  # noqa: F811
    bf16 = x.dtype == torch.bfloat16
    cut = plan.cut(x.shape[0], x.shape[1], bf16)
    tiles = -(-cut.tiles_per_split // cut.waves)
    c = ((16 if bf16 else 8) + 3) * tiles + 3 * (1 + 6 + 4 + 6) + 2 + 4 * E
    log_s = (lp.abs() if lp is not None else 0.0) + math.log(x.shape[1])  # (at least)
    return (c + 1 + 2 * log_s + 2 * (lp.abs() if lp is not None else 0.0)) * U, (c + 1 + 2 * E * c + 2 * math.log(x.shape[1]) + 2 * H) * U


SHAPES = [(1, 300001), (3, 128000), (3, 128001), (7, 50257), (100, 50257), (300, 20011), (515, 50021), (1030, 32003), (1030, 100003)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab", SHAPES)
@pytest.mark.parametrize("first,extra", [(0, 0), (1, 2), (5, 0)])
def test_equal_logits_are_counted_exactly(dtype, n, vocab, first, extra):
    """All exponentials are 1 and S is the vocabulary, exactly, so log S is off by its own evaluation: the instruction gives log2 S to
    one step, 2^-20 below 16 and 2^-19 from there on, which ln 2 is multiplied with, and the result is rounded by half a step of 2^-20
    between 8 and 16 (1.2 and 1.9 of these steps; 1.79 at 100003).  One logit more or less moves it by 1 / vocab."""
    x = rows_at(n, vocab, dtype, extra, first)
    x.fill_(1.5)
    t = torch.arange(n, device=DEV) % vocab
    lp, h, ids, top, stats = binding.bof4_token_logprobs(x, t, top=2)
    want = math.log(vocab)
    step = 1.01 * (math.log(2) * 2.0 ** (-20 if vocab < 1 << 16 else -19) + 2.0 ** -21)
    assert 1.0 / vocab > step and 8 < want < 16 and 8 <= math.log2(vocab) < 32
    assert bool(((lp.double() + want).abs() <= step).all()) and bool(((h.double() - want).abs() <= step).all())
    assert bool(((stats[:, 1].double() - want).abs() <= step).all()) and bool((stats[:, 0] == 1.5).all())
    assert bool((ids == torch.tensor([0, 1], device=DEV)).all())
    # without probability, one in each row: one fewer to count
    at = (torch.arange(n, device=DEV) * 7919 + vocab - 1) % vocab
    x[torch.arange(n, device=DEV), at] = -math.inf
    h = binding.bof4_token_logprobs(x)[1]
    assert bool(((h.double() - math.log(vocab - 1)).abs() <= step).all())


def seams(cut, vocab, per_word):
    """Ids at and around the ends of the row, of tiles and of parts, whatever a row's place in its first word."""
    ids = set(range(0, per_word + 2)) | set(range(vocab - per_word - 2, vocab))
    tiles = {1, 2, 3, cut.waves, cut.waves + 1, cut.tiles_per_split, 2 * cut.tiles_per_split, cut.splits * cut.tiles_per_split - 1,
             (cut.splits - 1) * cut.tiles_per_split, vocab // cut.tile, vocab // cut.tile - 1}
    for k in tiles:
        ids |= set(range(k * cut.tile - per_word - 1, k * cut.tile + 2))
    return sorted(i for i in ids if 0 <= i < vocab)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab", [(3, 128001), (90, 50257), (300, 20011), (515, 50021), (1030, 32003), (1030, 100003)])
def test_a_logit_that_dominates_at_every_seam(plan, dtype, n, vocab):  # noqa: F811
    bf16 = dtype == torch.bfloat16
    per_word = 8 if bf16 else 4
    ids = seams(plan.cut(n, vocab, bf16), vocab, per_word)
    g = torch.Generator(device=DEV).manual_seed(vocab)
    base = torch.randn((n, vocab + 1), generator=g, device=DEV).to(dtype)[:, :vocab]  # (odd strides: rows begin anywhere)
    ones = torch.ones(n, device=DEV)
    for i0 in range(0, len(ids), n):
        at = torch.tensor([ids[(i0 + r) % len(ids)] for r in range(n)], device=DEV)
        x = torch.empty((n, vocab + 1), dtype=dtype, device=DEV)[:, :vocab].copy_(base)
        x[torch.arange(n, device=DEV), at] = 14.0
        logp, p, H, E, want = reference(x, at)
        lp, h, top_ids, _, stats = binding.bof4_token_logprobs(x, at, top=3)
        b_lp, b_h = bounds(plan, x, E, want, H)
        assert bool(((lp.double() - want).abs() <= b_lp).all()) and bool(((h.double() - H).abs() <= b_h).all())
        assert bool((top_ids[:, 0] == at).all()) and bool((stats[:, 0] == 14.0).all())
        d = binding.bof4_token_logprobs_backward(x, stats, at, ones, h, ones, out_dtype=torch.float32).double()
        safe = torch.where(p > 0, logp, 0.0)
        exact = -p - p * (safe + H[:, None])
        exact.scatter_add_(1, at[:, None], torch.ones((n, 1), dtype=torch.float64, device=DEV))
        # p is off by log p's error relatively, and the products by a few roundings
        rel = b_lp[:, None] + b_h[:, None] + (4 * safe.abs() + 8) * U
        assert bool(((d - exact).abs() <= p * (1 + safe.abs() + H[:, None]) * rel + 4 * U * exact.abs() + 2.0 ** -126).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab", SHAPES + [(2, 4097), (40, 32000), (700, 3001)])
@pytest.mark.parametrize("spread", [0.3, 3.0])
def test_sums_within_the_chain_that_a_lane_adds(plan, dtype, n, vocab, spread):  # noqa: F811
    g = torch.Generator(device=DEV).manual_seed(n + vocab)
    x = (spread * torch.randn((n, vocab), generator=g, device=DEV)).to(dtype)
    t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    _, _, H, E, want = reference(x, t)
    lp, h, _, _, _ = binding.bof4_token_logprobs(x, t)
    b_lp, b_h = bounds(plan, x, E, want, H)
    assert bool(((lp.double() - want).abs() <= b_lp).all()), float(((lp.double() - want).abs() / b_lp).max())
    assert bool(((h.double() - H).abs() <= b_h).all()), float(((h.double() - H).abs() / b_h).max())
