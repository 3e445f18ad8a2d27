"""The gradient by x of a linear layer where the caller's tensors are binary32: dz goes into the sums in as many bfloat16 terms as
the tensors call for, and not in one.

Bounds, U = 2^-24.  dz itself is off by 32 U (1 + |z|) of dy * mul under an activation and by 2 U of itself without one (as in
test_gpu_linear).  A term leaves at most 2^-8 of what it rounds: dz in two terms is off by 2^-16 of itself, in three by 2^-24.  The
sums are of up to three terms per row: (3 rows + 64) U of sum |dz w|.  A result in bfloat16 is rounded by 2^-8 of itself."""
import math

import pytest
import torch

from paper_2505_06653_amd import binding
from test_gpu_linear import ACTS, DEV, U, Matrix, act64, half_step, randn

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# one token and many, rows and columns that end inside tiles, rows shared by several workgroups and not, workgroups of 192 and
# of 256 columns, several slabs, dz made apart from the turned matrix and with it
SHAPES = [(1, 32, 1, 0.0), (3, 64, 5, 0.1), (65, 96, 40, 0.05), (100, 2080, 33, 0.02), (1001, 1504, 300, 0.0), (33, 32768, 40, 0.001),
          (16390, 128, 70, 0.01), (4111, 4128, 333, 0.006), (2050, 2080, 2001, 0.003), (70001, 160, 100, 0.01), (9000, 16384, 130, 0.002),
          (1376, 4096, 129, 0.0)]


def gradient(m, n_tokens, act, dy, mul, out, seed=5):
    """dx, what it should be, the allowed error without dz's own terms, and sum |dz w|."""
    shape = (n_tokens, m.rows)
    g = randn(shape, seed, dy)
    args = {"act": act, "out_dtype": out}
    if act != "none":
        args["pre"] = randn(shape, seed + 1, F32)
    if mul is not None:
        args["mul"] = randn(shape, seed + 2, mul)
    dx = m.backward(g, **args)
    z = args["pre"].double() if act != "none" else torch.zeros(shape, dtype=torch.float64, device=DEV)
    dz = g.double() * (args["mul"].double() if mul is not None else 1.0)
    err = (32 * U * (1 + z.abs()) if act != "none" else 2 * U) * dz.abs()
    dz = dz * act64(act, z)[1]
    w = m.gemm_w.abs()
    want, size = dz @ m.gemm_w, dz.abs() @ w
    return dx, want, ((3 * m.rows + 64) * U * size + err @ w + half_step(want, out)) * 1.01, size


@pytest.mark.parametrize("rows,cols,n_tokens,share", SHAPES)
def test_binary32_results_take_dz_in_binary32(rows, cols, n_tokens, share):
    m = Matrix(rows, cols, share)
    for act, dy, mul in (("silu", BF16, BF16), ("gelu", F32, F32), ("none", F32, None), ("none", BF16, BF16), ("relu", BF16, None)):
        dx, want, tol, size = gradient(m, n_tokens, act, dy, mul, F32)
        off = (dx.double() - want).abs()
        assert bool((off <= tol + U * size).all()), (act, float((off / (tol + U * size)).max()))
        # roundings are independent of each other: together they stay below a chain of 512 terms' bound
        assert float(off.square().mean().sqrt()) <= 512 * U * float(size.square().mean().sqrt())


@pytest.mark.parametrize("rows,cols,n_tokens,share", SHAPES)
def test_bfloat16_results_of_binary32_gradients_take_dz_in_sixteen_bits(rows, cols, n_tokens, share):
    m = Matrix(rows, cols, share)
    for act, mul in (("silu", BF16), ("none", None), ("gelu_tanh", F32)):
        dx, want, tol, size = gradient(m, n_tokens, act, F32, mul, BF16)
        off = (dx.double() - want).abs()
        assert bool((off <= tol + 2.0 ** -16 * size).all()), (act, float((off / (tol + 2.0 ** -16 * size)).max()))


@pytest.mark.parametrize("act", ACTS)
def test_activations_in_binary32(act):
    dx, want, tol, size = gradient(Matrix(130, 96, 0.02), 70, act, F32, F32, F32)
    assert bool(((dx.double() - want).abs() <= tol + U * size).all())


def test_gradients_that_are_not_finite_stay_with_their_token():
    """What the first term cannot hold leaves nothing for the others: no NaN out of an infinite or very large dz."""
    m = Matrix(130, 96)
    dy = randn((9, 130), 1, F32)
    want = m.backward(dy, out_dtype=F32)
    row, cols = 4, m.gemm_w[4] != 0  # (0 times infinity is NaN)
    keep = [0, 1, 2, 3, 5, 6, 7, 8]
    for value in (math.inf, -math.inf, 3.4e38, -3.4e38):
        bad = dy.clone()
        bad[4, row] = value
        got = m.backward(bad, out_dtype=F32)
        assert torch.equal(got[keep], want[keep]) and not bool(got[4][cols].isnan().any())
        if math.isinf(value):
            assert torch.equal(got[4][cols].double(), value * m.gemm_w[row][cols])
    bad[4, row] = math.nan
    got = m.backward(bad, out_dtype=F32)
    assert torch.equal(got[keep], want[keep]) and bool(got[4].isnan().all())


def test_equal_bits_captured_and_in_a_workspace_of_the_stated_size():
    rows, cols, n_tokens = 1001, 2080, 300
    m = Matrix(rows, cols, 0.01)
    dy, pre = randn((n_tokens, rows), 1, F32), randn((n_tokens, rows), 2, F32)
    size = binding.bof4_gemm_linear_backward_workspace_bytes(rows, cols, n_tokens)
    whole = torch.full((size + 4096,), 0xff, dtype=torch.uint8, device=DEV)
    for out in (F32, BF16):
        want = m.backward(dy, act="silu", pre=pre, out_dtype=out)
        held, dx = dy.clone(), torch.empty((n_tokens, cols), dtype=out, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.backward(held, act="silu", pre=pre, out=dx, ws=whole[:size])
        for k in range(3):
            held.copy_(torch.roll(dy, k, 0))
            dx.fill_(math.nan)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dx, m.backward(torch.roll(dy, k, 0), act="silu", pre=pre, out_dtype=out))
        assert torch.equal(m.backward(dy, act="silu", pre=pre, out_dtype=out), want) and bool((whole[size:] == 0xff).all())


def test_tokens_in_several_passes():
    """More tokens than dz's three terms have room for at once (4 GiB): tokens of every pass and around their borders, and dbias of
    all of them, against binary64; what is written over dy on the way is dmul."""
    rows, cols, n_tokens = 1 << 18, 96, 5500  # passes of 2688, 2688 and 124 tokens
    m = Matrix(rows, cols, 0.0005)
    shape = (n_tokens, rows)
    dy = torch.empty(shape, dtype=F32, device=DEV)
    pre, mul = torch.empty(shape, dtype=BF16, device=DEV), torch.empty(shape, dtype=BF16, device=DEV)
    for t in range(0, n_tokens, 500):
        dy[t:t + 500], pre[t:t + 500], mul[t:t + 500] = (randn((500, rows), 10 * t + k, F32) for k in range(3))
    picked = torch.tensor([0, 1, 2687, 2688, 2689, 5375, 5376, 5499], device=DEV)
    z, f, g = pre[picked].double(), mul[picked].double(), dy[picked].double()
    a, slope = act64("silu", z)
    dz, err = g * f * slope, 32 * U * (1 + z.abs()) * (g * f).abs()
    total, total_abs = torch.zeros(rows, dtype=torch.float64, device=DEV), torch.zeros(rows, dtype=torch.float64, device=DEV)
    for t in range(0, n_tokens, 500):
        part = dy[t:t + 500].double() * mul[t:t + 500].double()
        total_abs += part.abs().mul_(1 + pre[t:t + 500].double().abs()).sum(0)
        total += part.mul_(act64("silu", pre[t:t + 500].double())[1]).sum(0)
    dbias = torch.full((rows,), math.nan, device=DEV)
    dx = m.backward(dy, act="silu", pre=pre, mul=mul, dmul=dy, dbias=dbias, out_dtype=F32)
    w = m.gemm_w.abs()
    want, size = dz @ m.gemm_w, dz.abs() @ w
    assert bool(((dx[picked].double() - want).abs() <= 1.01 * ((3 * rows + 65) * U * size + err @ w + half_step(want, F32))).all())
    # (and as a whole well below the bound of such long sums: a term of one token lost or taken twice shows)
    assert float((dx[picked].double() - want).square().mean().sqrt()) <= 512 * U * float(size.square().mean().sqrt())
    assert bool(((dy[picked].double() - g * a).abs() <= (32 * U * (1 + z.abs()) + 2 * U * a.abs()) * g.abs() + 1.01 * half_step(g * a, F32)).all())
    # slopes are below 1.2 and off by 32 U (1 + |z|); 5500 binary32 additions in chains of 1 + 32 (and binary64)
    assert bool(((dbias.double() - total).abs() <= (32 + 1.2 * 64 + 2) * U * total_abs).all())


@pytest.mark.parametrize("rows,cols,n_tokens", [(1001, 96, 9), (100, 2080, 33), (520, 512, 300), (4111, 160, 2000)])
@pytest.mark.parametrize("first,extra", [(0, 0), (1, 2), (4, 4)])
def test_rows_of_any_stride_over_its_own_inputs_and_nothing_else_is_written(rows, cols, n_tokens, first, extra):
    m = Matrix(rows, cols, 0.01)

    def inside(width, dtype, seed, fill=None):
        whole = randn((n_tokens + 2, first + width + extra), seed, dtype)
        if fill is not None:
            whole.fill_(fill)
        return whole, whole[1:-1, first:first + width]

    (_, dy), (_, pre), (_, mul) = inside(rows, F32, 1), inside(rows, BF16, 2), inside(rows, F32, 3)
    dmul = torch.empty((n_tokens, rows), device=DEV)
    want = m.backward(dy.contiguous(), act="silu", pre=pre.contiguous(), mul=mul.contiguous(), dmul=dmul, out_dtype=F32)
    whole, dx = inside(cols, F32, 4, 7.0)
    m.backward(dy, act="silu", pre=pre, mul=mul, out=dx)
    assert torch.equal(dx, want)
    whole[1:-1, first:first + cols] = 7.0
    assert bool((whole == 7.0).all())
    for over in ("dy", "mul"):
        t = {"dy": dy.clone(), "mul": mul.clone()}
        assert torch.equal(m.backward(t["dy"], act="silu", pre=pre, mul=t["mul"], dmul=t[over], out_dtype=F32), want)
        assert torch.equal(t[over], dmul)


def test_calls_with_other_types_side_by_side():
    """One, two and three terms at the same time on streams of their own: what each gives alone."""
    m, n = Matrix(4111, 2080, 0.01), 300
    dys = [randn((n, 4111), 1, BF16), randn((n, 4111), 2, F32), randn((n, 4111), 3, F32)]
    outs = [BF16, BF16, F32]
    want = [m.backward(dy, out_dtype=out) for dy, out in zip(dys, outs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in outs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[m.backward(dy, out_dtype=out, stream=s) for dy, out, s in zip(dys, outs, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for one in got for a, b in zip(one, want))
