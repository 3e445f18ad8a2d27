"""The linear layer around the products (bof4_gemv_linear, bof4_gemm_linear) and its gradients against binary64.

Bounds, U = 2^-24.  The sums z are those of the products: within 64 U (gemv) or (cols + 64) U (gemm) of sum |w x|.  Behind them:
one rounding per operation; an activation's slope is below 1.2, and its own evaluation (an exponential or error function of a
few U, a reciprocal, three products) is off by at most 32 U (1 + |z|).  A result in bfloat16 is rounded once, by half a step at
most: 2^-8 of its value.  In the gradients dz is rounded to bfloat16 where there is an activation or a factor: 2^-8 of each term
of the sums, which are otherwise within (rows + 64) U of sum |dz w|."""
import math

import numpy as np
import pytest
import torch

from paper_2505_06653_amd import binding
from test_gpu_parity import cb_for
from test_host_gemm_plan import DECODED, NARROW, WIDE, rules  # noqa: F401 (a fixture: the host's choice of the kernel)

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
ACTS = list(binding.ACTIVATIONS)


class Matrix:
    """A quantised matrix with everything that the calls take, and its weights in binary64 for either product."""

    def __init__(self, rows, cols, share=0.0, block=32, seed=0):
        g = torch.Generator(device=DEV).manual_seed(1000 * seed + rows + cols)
        n = rows * cols
        self.rows, self.cols, self.block = rows, cols, block
        self.codes = torch.randint(0, 256, (n // 2,), generator=g, device=DEV, dtype=torch.uint8)
        self.scales = ((torch.rand(n // block, generator=g, device=DEV) - 0.5) * 0.2).to(torch.float16)
        self.cb = cb_for(block, 1)
        self.k, oi, ov, self.gemv_table, self.gemm_table = int(n * share), None, None, None, None
        if self.k:
            oi = torch.unique(torch.randint(0, n, (self.k,), generator=g, device=DEV))
            self.k = oi.numel()
            ov = torch.randn(self.k, generator=g, device=DEV).to(torch.float16)
            args = (self.codes, self.scales, rows, cols, block, self.cb, oi, ov)
            self.gemv_table = binding.bof4_gemv_outlier_table(*args)
            self.gemm_table = binding.bof4_gemm_outlier_table(*args)
        self.packed = binding.bof4_gemm_pack(self.codes, self.scales, rows, cols, block)
        lv = torch.tensor(self.cb, device=DEV).float().double()
        nibbles = torch.stack((self.codes % 16, self.codes // 16), 1).reshape(-1, block).long()
        w = lv[nibbles] * self.scales.double()[:, None]
        self.gemm_w = binding.bof4_dequantize(self.codes, self.scales, n, block, self.cb, oi, ov).reshape(rows, cols).double()
        self.gemv_w, self.placeholders = w.reshape(-1).clone(), torch.zeros(n, dtype=torch.float64, device=DEV)
        if self.k:
            self.placeholders[oi] = self.gemv_w[oi].abs()
            self.gemv_w[oi] = ov.double()
        self.gemv_w, self.placeholders = self.gemv_w.reshape(rows, cols), self.placeholders.reshape(rows, cols)

    def linear(self, way, x, **kw):
        if way == "gemv":
            return binding.bof4_gemv_linear(self.codes, self.scales, self.rows, self.cols, self.block, self.cb, x, self.gemv_table,
                                            self.k, **kw)
        return binding.bof4_gemm_linear(self.packed, self.rows, self.cols, self.cb, x, self.gemm_table, self.k, **kw)

    def product(self, way, x):
        if way == "gemv":
            return binding.bof4_gemv(self.codes, self.scales, self.rows, self.cols, self.block, self.cb, x, self.gemv_table, self.k)
        return binding.bof4_gemm(self.packed, self.rows, self.cols, self.cb, x, self.gemm_table, self.k)

    def backward(self, dy, **kw):
        return binding.bof4_gemm_linear_backward(self.packed, self.rows, self.cols, self.cb, dy, self.gemm_table, self.k, **kw)


def randn(shape, seed, dtype=torch.bfloat16, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(shape, generator=g, device=DEV)).to(dtype)


def act64(act, z):
    """The activation and, by differentiation, its slope."""
    z = z.detach().clone().requires_grad_(True)
    a = {"none": lambda: z * 1.0, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.ndtr(z),
         "gelu_tanh": lambda: 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))),
         "silu": lambda: z * torch.sigmoid(z)}[act]()
    slope, = torch.autograd.grad(a.sum(), z)
    return a.detach(), slope


def half_step(t, dtype):
    return t.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else U) + 2.0 ** -133


def check(m, way, n_tokens, act="none", bias=None, mul=None, residual=None, pre=None, out=torch.bfloat16, seed=1, **kw):
    """bias, mul, residual, pre: types, or None."""
    shape = (n_tokens, m.rows)
    x = randn((n_tokens, m.cols), seed)
    args = {"act": act, "out_dtype": out}
    if bias is not None:
        args["bias"] = randn(m.rows, seed + 1, bias)
    if mul is not None:
        args["mul"] = randn(shape, seed + 2, mul)
    if residual is not None:
        args["residual"] = randn(shape, seed + 3, residual)
    if pre is not None:
        args["pre"] = torch.full(shape, math.nan, dtype=pre, device=DEV)
    y = m.linear(way, x, **args, **kw)
    w = m.gemv_w if way == "gemv" else m.gemm_w
    z = x.double() @ w.t().contiguous()
    size = x.double().abs() @ (w.abs() + (m.placeholders if way == "gemv" else 0)).t().contiguous()
    err = (64 if way == "gemv" else m.cols + 64) * U * size
    if bias is not None:
        z = z + args["bias"].double()
        err = err + 2 * U * z.abs()
    if pre is not None:
        assert bool(((args["pre"].double() - z).abs() <= err * 1.01 + half_step(z, pre)).all())
    a = act64(act, z)[0]
    err = 1.2 * err + (32 * U * (1 + z.abs()) if act != "none" else 0)
    if mul is not None:
        a, err = a * args["mul"].double(), err * args["mul"].double().abs()
        err = err + U * a.abs()
    if residual is not None:
        a = a + args["residual"].double()
    err = err + 2 * U * a.abs() + half_step(a, out) * 1.01
    assert y.dtype == out and y.shape == shape
    worst = float(((y.double() - a).abs() / (err + 1e-30)).max())
    assert worst <= 1.0, worst
    return x, args, y


GEMV = [(1, 32, 1, 0.0), (37, 96, 2, 0.05), (1001, 1504, 3, 0.0), (130, 2080, 1, 0.02), (70, 6144, 4, 0.01), (300, 16416, 1, 0.0),
        (5000, 512, 5, 0.01), (9, 32768, 7, 0.0), (4100, 4128, 1, 0.006)]


@pytest.mark.parametrize("rows,cols,n_tokens,share", GEMV)
@pytest.mark.parametrize("act", ACTS)
def test_gemv_linear(rows, cols, n_tokens, share, act):
    m = Matrix(rows, cols, share)
    bf16, f32 = torch.bfloat16, torch.float32
    check(m, "gemv", n_tokens, act, bias=bf16, residual=bf16)
    check(m, "gemv", n_tokens, act, bias=f32, mul=bf16, residual=f32, pre=f32, out=f32)
    check(m, "gemv", n_tokens, act, mul=f32, pre=bf16)


# ways: x read in place, split columns, two row tiles a wave, the 256 x 128 tile whole and split, decoded first whole and split
GEMM = [(1, 32, 1, 0.0, NARROW), (3, 64, 5, 0.1, NARROW), (70, 1536, 33, 0.02, NARROW), (33, 32768, 40, 0.001, NARROW),
        (16390, 128, 70, 0.01, NARROW), (8200, 2080, 6, 0.0, NARROW), (8200, 2080, 6, 0.01, NARROW), (12320, 2304, 130, 0.005, NARROW),
        (300, 2304, 330, 0.01, WIDE), (521, 512, 600, 0.0, WIDE), (1001, 1504, 300, 0.006, WIDE), (300, 4096, 400, 0.0, WIDE),
        (4111, 4128, 1001, 0.006, DECODED), (2050, 2080, 2001, 0.0, DECODED), (500, 28672, 400, 0.01, DECODED),
        (4099, 8224, 900, 0.006, DECODED)]


@pytest.mark.parametrize("rows,cols,n_tokens,share,way", GEMM)
def test_gemm_linear(rules, rows, cols, n_tokens, share, way):
    assert rules(rows, cols, n_tokens, share > 0).way == way
    m = Matrix(rows, cols, share)
    bf16, f32 = torch.bfloat16, torch.float32
    check(m, "gemm", n_tokens, "none", bias=bf16)
    check(m, "gemm", n_tokens, "none", residual=f32, out=f32)
    check(m, "gemm", n_tokens, "silu", mul=bf16, pre=bf16)
    check(m, "gemm", n_tokens, "gelu", bias=f32, mul=f32, residual=bf16, pre=f32, out=f32)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,cols,n_tokens", [(65, 96, 40), (300, 2304, 330)])
def test_gemm_linear_activations(rows, cols, n_tokens, act):
    check(Matrix(rows, cols, 0.01), "gemm", n_tokens, act, bias=torch.bfloat16, residual=torch.bfloat16, out=torch.float32)


@pytest.mark.parametrize("rows,cols,n_tokens,share,way", GEMM)
def test_empty_layer_is_the_product_bit_for_bit(rows, cols, n_tokens, share, way):
    m = Matrix(rows, cols, share)
    x = randn((n_tokens, cols), 4)
    assert torch.equal(m.linear("gemm", x, out_dtype=torch.float32), m.product("gemm", x))


@pytest.mark.parametrize("rows,cols,n_tokens,share", GEMV)
def test_empty_layer_is_the_vector_product_bit_for_bit(rows, cols, n_tokens, share):
    m = Matrix(rows, cols, share)
    x = randn((n_tokens, cols), 4)
    y = m.product("gemv", x)
    assert torch.equal(m.linear("gemv", x, out_dtype=torch.float32), y)
    assert torch.equal(m.linear("gemv", x), y.to(torch.bfloat16))


LAYOUTS = [("gemv", 1001, 96, 3), ("gemm", 1001, 96, 9), ("gemm", 70, 1536, 33), ("gemm", 300, 2304, 330), ("gemm", 521, 512, 600),
           ("gemm", 4111, 4128, 600)]


@pytest.mark.parametrize("way,rows,cols,n_tokens", LAYOUTS)
@pytest.mark.parametrize("first,extra", [(0, 0), (1, 2), (4, 4)])
def test_rows_of_any_stride_and_nothing_else_is_written(way, rows, cols, n_tokens, first, extra):
    m = Matrix(rows, cols, 0.01)
    x = randn((n_tokens, cols), 1)

    def inside(dtype, seed, fill=None):  # rows with `first` elements in front and `extra` behind, tokens around
        whole = randn((n_tokens + 2, first + rows + extra), seed, dtype)
        if fill is not None:
            whole.fill_(fill)
        return whole, whole[1:-1, first:first + rows]

    _, mul = inside(torch.bfloat16, 2)
    _, residual = inside(torch.float32, 3)
    whole_y, y = inside(torch.bfloat16, 4, 7.0)
    whole_z, z = inside(torch.float32, 5, 7.0)
    m.linear(way, x, act="gelu_tanh", mul=mul, residual=residual, pre=z, out=y)
    pre = torch.empty((n_tokens, rows), device=DEV)
    want = m.linear(way, x, act="gelu_tanh", mul=mul.contiguous(), residual=residual.contiguous(), pre=pre)
    assert torch.equal(y, want) and torch.equal(z, pre)
    for whole in (whole_y, whole_z):
        whole[1:-1, first:first + rows] = 7.0
        assert bool((whole == 7.0).all())


@pytest.mark.parametrize("way,rows,cols,n_tokens", LAYOUTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_result_over_the_residual_and_over_the_factor(way, rows, cols, n_tokens, dtype):
    m = Matrix(rows, cols, 0.01)
    x, r = randn((n_tokens, cols), 1), randn((n_tokens, rows), 2, dtype)
    want = m.linear(way, x, residual=r, out_dtype=dtype)
    stream = r.clone()
    assert m.linear(way, x, residual=stream, out=stream) is stream and torch.equal(stream, want)
    want = m.linear(way, x, act="silu", mul=r, out_dtype=dtype)
    stream = r.clone()
    m.linear(way, x, act="silu", mul=stream, out=stream)
    assert torch.equal(stream, want)


@pytest.mark.parametrize("way,rows,cols,n_tokens", LAYOUTS)
def test_a_token_that_is_not_finite_stays_on_its_own(way, rows, cols, n_tokens):
    m = Matrix(rows, cols, 0.01)
    x, r = randn((n_tokens, cols), 1), randn((n_tokens, rows), 2)
    want = m.linear(way, x, act="silu", residual=r)
    bad = n_tokens // 2
    x[bad, 3] = math.nan
    got = m.linear(way, x, act="silu", residual=r)
    keep = [t for t in range(n_tokens) if t != bad]
    assert torch.equal(got[keep], want[keep]) and bool(got[bad].isnan().all())
    r[0, 1], r[0, 2] = math.inf, math.nan  # a residual's, too
    x[bad, 3] = 0.0
    got = m.linear(way, x, act="silu", residual=r)
    assert got[0, 1] == math.inf and got[0, 2].isnan() and int((~got.isfinite()).sum()) == 2


def test_activations_far_out():
    """z picked through a bias: no NaN and no loss of the limits where exponentials overflow or vanish."""
    m = Matrix(64, 32)
    x = torch.zeros((1, 32), dtype=torch.bfloat16, device=DEV)
    z = torch.cat((-torch.logspace(-30, 30, 31), torch.logspace(-30, 30, 31), torch.zeros(2))).to(DEV)
    for act in ACTS:
        for way in ("gemv", "gemm"):
            y = m.linear(way, x, bias=z, act=act, out_dtype=torch.float32)[0]
            want = act64(act, z.double())[0]
            want = torch.where(want.isnan(), torch.where(z > 0, z, 0.0).double(), want)
            assert bool(((y.double() - want).abs() <= 32 * U * want.abs() + 32 * U * torch.clamp(z.abs(), max=30.0).double()).all()), act
            d = m.backward(torch.ones((1, 64), device=DEV), act=act, pre=z[None, :], out_dtype=torch.float32)
            assert bool(d.isfinite().all()), act


# ------------------------------------------------------------------------------------------------ gradients
# dz with the turned matrix and apart from it, one slab and two, rows split and not
GRAD = [(1, 32, 1, 0.0), (70001, 160, 100, 0.01), (3, 64, 5, 0.1), (65, 96, 40, 0.05), (100, 2080, 33, 0.02), (1001, 1504, 300, 0.0), (33, 32768, 40, 0.001),
        (16390, 128, 70, 0.01), (4111, 4128, 333, 0.006), (2050, 2080, 2001, 0.003), (70001, 160, 9, 0.01), (9000, 16384, 130, 0.002),
        (64, 224, 130, 0.9)]


def check_grad(m, n_tokens, act, mul=None, dmul=None, dbias=False, dy=torch.bfloat16, pre=torch.bfloat16, out=torch.bfloat16, seed=5):
    shape = (n_tokens, m.rows)
    g = randn(shape, seed, dy)
    args = {"act": act, "out_dtype": out}
    if act != "none" or dmul is not None:
        args["pre"] = randn(shape, seed + 1, pre)
    if mul is not None:
        args["mul"] = randn(shape, seed + 2, mul)
    if dmul is not None:
        args["dmul"] = torch.full(shape, math.nan, dtype=dmul, device=DEV)
    if dbias:
        args["dbias"] = torch.full((m.rows,), math.nan, device=DEV)
    dx = m.backward(g, **args)
    z = args["pre"].double() if "pre" in args else torch.zeros(shape, dtype=torch.float64, device=DEV)
    a, slope = act64(act, z)
    dz = g.double() * (args["mul"].double() if mul is not None else 1.0)
    err = 32 * U * (1 + z.abs()) * dz.abs() if act != "none" else 2 * U * dz.abs()
    dz = dz * slope
    if dmul is not None:
        want = g.double() * a
        tol = (32 * U * (1 + z.abs()) + 2 * U * a.abs()) * g.double().abs() + half_step(want, dmul) * 1.01
        assert bool(((args["dmul"].double() - want).abs() <= tol).all())
    if dbias:
        tol = (n_tokens + 64) * U * dz.abs().sum(0) + err.sum(0) + 1e-37
        assert bool(((args["dbias"].double() - dz.sum(0)).abs() <= tol).all())
    exact = act == "none" and mul is None and dy == torch.bfloat16
    w = m.gemm_w
    want, size = dz @ w, dz.abs() @ w.abs()
    tol = (m.rows + 64) * U * size * 1.01 + half_step(want, out) * 1.01
    if not exact:
        tol = tol + 2.0 ** -8 * size + err @ w.abs()
    assert dx.dtype == out and bool(((dx.double() - want).abs() <= tol).all()), float(((dx.double() - want).abs() / tol).max())
    # the roundings of dz are independent of each other: together well below their bound
    rms, scale = (dx.double() - want).square().mean().sqrt(), (dz.square() @ w.square()).mean().sqrt()
    assert float(rms) <= 2.0 ** -8 * float(scale) + float(half_step(want, out).square().mean().sqrt())
    return g, args, dx


@pytest.mark.parametrize("rows,cols,n_tokens,share", GRAD)
def test_gradients(rows, cols, n_tokens, share):
    m = Matrix(rows, cols, share)
    bf16, f32 = torch.bfloat16, torch.float32
    check_grad(m, n_tokens, "none", out=f32)
    check_grad(m, n_tokens, "none", dbias=True)
    check_grad(m, n_tokens, "silu", mul=bf16, dmul=bf16, dbias=True)
    check_grad(m, n_tokens, "gelu", mul=f32, dmul=f32, dy=f32, pre=f32, out=f32)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_of_the_activations(act):
    check_grad(Matrix(130, 96, 0.02), 70, act, mul=torch.bfloat16, dmul=torch.float32, dbias=True)


def test_gradient_against_differences():
    """sum(dy * y) of the forward call, its residual left out, moved by one input at a time: central differences of binary64 at
    step h, whose own error is of the order h^2."""
    m = Matrix(33, 64, 0.05)
    x = randn((4, 64), 1, torch.float64)
    bias, mul, dy = randn(33, 2, torch.float32), randn((4, 33), 3, torch.float32), randn((4, 33), 4, torch.bfloat16)
    pre = (x @ m.gemm_w.t() + bias.double()).float()
    dmul, dbias = torch.empty((4, 33), device=DEV), torch.empty(33, device=DEV)
    dx = m.backward(dy, act="gelu_tanh", pre=pre, mul=mul, dmul=dmul, dbias=dbias, out_dtype=torch.float32)

    def loss(x, bias, mul):
        return (dy.double() * act64("gelu_tanh", x @ m.gemm_w.t() + bias)[0] * mul).sum()

    h, base = 1e-5, [x, bias.double(), mul.double()]
    for which, grad in ((0, dx), (1, dbias), (2, dmul)):
        flat = grad.reshape(-1)
        for at in range(0, flat.numel(), max(1, flat.numel() // 40)):
            moved = []
            for sign in (1, -1):
                args = [b.clone() for b in base]
                args[which].view(-1)[at] += sign * h
                moved.append(loss(*args))
            diff = float((moved[0] - moved[1]) / (2 * h))
            # dz in bfloat16: 2^-8 of the terms' sum for dx
            slack = 2.0 ** -8 * float((dy.double().abs() * 1.2 * mul.double().abs()) [at // 64].abs() @ m.gemm_w[:, at % 64].abs()) if which == 0 else 0
            assert abs(float(flat[at]) - diff) <= 1e-5 * (1 + abs(diff)) + slack, (which, at)


@pytest.mark.parametrize("rows,cols,n_tokens", [(1001, 96, 9), (100, 2080, 33), (520, 512, 300)])
@pytest.mark.parametrize("first,extra", [(0, 0), (1, 2), (4, 4)])
def test_gradients_rows_of_any_stride_and_nothing_else_is_written(rows, cols, n_tokens, first, extra):
    m = Matrix(rows, cols, 0.01)

    def inside(width, dtype, seed, fill=None):
        whole = randn((n_tokens + 2, first + width + extra), seed, dtype)
        if fill is not None:
            whole.fill_(fill)
        return whole, whole[1:-1, first:first + width]

    _, dy = inside(rows, torch.bfloat16, 1)
    _, pre = inside(rows, torch.float32, 2)
    _, mul = inside(rows, torch.bfloat16, 3)
    whole_dx, dx = inside(cols, torch.bfloat16, 4, 7.0)
    whole_dm, dm = inside(rows, torch.bfloat16, 5, 7.0)
    m.backward(dy, act="silu", pre=pre, mul=mul, dmul=dm, out=dx)
    dmul = torch.empty((n_tokens, rows), dtype=torch.bfloat16, device=DEV)
    want = m.backward(dy.contiguous(), act="silu", pre=pre.contiguous(), mul=mul.contiguous(), dmul=dmul)
    assert torch.equal(dx, want) and torch.equal(dm, dmul)
    whole_dx[1:-1, first:first + cols] = 7.0
    whole_dm[1:-1, first:first + rows] = 7.0
    assert bool((whole_dx == 7.0).all()) and bool((whole_dm == 7.0).all())
    for name, t in (("dy", dy), ("mul", mul)):  # over its own inputs
        t2 = t.contiguous().clone()
        a = {"dy": dy.contiguous(), "mul": mul.contiguous(), name: t2}
        assert torch.equal(m.backward(a["dy"], act="silu", pre=pre.contiguous(), mul=a["mul"], dmul=t2), want) and torch.equal(t2, dmul)


def test_gradient_picks_single_decoded_weights():
    """dz = unit vectors: every weight of the turned matrix comes out alone, in its place, exactly."""
    for rows, cols, share in ((70, 160, 0.0), (130, 96, 0.3), (257, 2080, 0.02)):
        m = Matrix(rows, cols, share)
        dx = m.backward(torch.eye(rows, dtype=torch.bfloat16, device=DEV), out_dtype=torch.float32)
        assert torch.equal(dx.double(), m.gemm_w)


@pytest.mark.parametrize("rows,cols,n_tokens", [(1001, 96, 40), (300, 8192, 300), (4111, 4128, 600)])
def test_equal_bits_streams_workspaces_and_captured(rows, cols, n_tokens):
    m = Matrix(rows, cols, 0.01)
    x, mul, dy = randn((n_tokens, cols), 1), randn((n_tokens, rows), 2), randn((n_tokens, rows), 3)

    def new():
        return {k: torch.empty((n_tokens, rows), dtype=torch.bfloat16, device=DEV) for k in ("pre", "dmul")}

    def both(x, buf, y=None, dx=None, ws=(None, None), stream=None):
        dbias = buf.setdefault("dbias", torch.empty(rows, device=DEV))
        y = m.linear("gemm", x, act="silu", mul=mul, pre=buf["pre"], out=y, ws=ws[0], stream=stream)
        dx = m.backward(dy, act="silu", pre=buf["pre"], mul=mul, dmul=buf["dmul"], dbias=dbias, out=dx, ws=ws[1], stream=stream)
        return [y, buf["pre"], dx, buf["dmul"], dbias]

    first = [t.clone() for t in both(x, new())]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    second = both(x, new(), stream=s)
    s.synchronize()
    sizes = (binding.bof4_gemm_linear_workspace_bytes(rows, cols, n_tokens), binding.bof4_gemm_linear_backward_workspace_bytes(rows, cols, n_tokens))
    whole = [torch.full((size + 4096,), 0xff, dtype=torch.uint8, device=DEV) for size in sizes]
    third = both(x, new(), ws=[w[:size] for w, size in zip(whole, sizes)])
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert all(bool((w[size:] == 0xff).all()) for w, size in zip(whole, sizes))
    more = both(x, new(), ws=[torch.empty(f(rows, cols, n_tokens + 700), dtype=torch.uint8, device=DEV) for f in (
        binding.bof4_gemm_linear_workspace_bytes, binding.bof4_gemm_linear_backward_workspace_bytes)])
    for a, b in zip(first, more):
        assert torch.equal(a, b)
    xs, buf, ws = x.clone(), new(), [w[:size] for w, size in zip(whole, sizes)]
    both(xs, buf, ws=ws)  # (occupancy is asked for once)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both(xs, buf, ws=ws)
    for k in range(3):
        xs.copy_(torch.roll(x, k, 0))
        graph.replay()
        torch.cuda.synchronize()
        want = both(torch.roll(x, k, 0), new())
        for a, b in zip(captured, want):
            assert torch.equal(a, b)


def test_two_calls_side_by_side_on_two_streams():
    """Each with a workspace of its own, forward and back, while the other runs: what each gives alone."""
    shapes = [(4111, 4128, 300), (1001, 2080, 600)]
    ms = [Matrix(r, c, 0.01) for r, c, _ in shapes]
    xs = [randn((n, c), 1) for _, c, n in shapes]
    dys = [randn((n, r), 2) for r, _, n in shapes]

    def run(i, stream=None):
        y = ms[i].linear("gemm", xs[i], act="relu", stream=stream)
        v = ms[i].linear("gemv", xs[i][:3].contiguous(), act="relu", stream=stream)
        return y, v, ms[i].backward(dys[i], stream=stream)

    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[run(i, streams[i]) for i in range(2)] for _ in range(4)]
    torch.cuda.synchronize()
    for round_ in got:
        for a, b in zip(round_, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_least_workspace_takes_another_way_and_less_is_refused():
    rows, cols, n_tokens = 2050, 2080, 2001
    m = Matrix(rows, cols, 0.003)
    x = randn((n_tokens, cols), 1)
    want = m.linear("gemm", x, out_dtype=torch.float32)
    size = m.gemm_w.abs()
    least = 4 * ((n_tokens + 31) // 32 * 32) * ((cols + 63) // 64 * 64) + 4 * 128 * rows * 64
    ws = torch.empty(min(least, binding.bof4_gemm_linear_workspace_bytes(rows, cols, n_tokens)), dtype=torch.uint8, device=DEV)
    got = m.linear("gemm", x, out_dtype=torch.float32, ws=ws)
    assert bool(((got - want).double().abs() <= 2 * (cols + 64) * U * (x.double().abs() @ size.t())).all())
    with pytest.raises(binding.Bof4Error):
        m.linear("gemm", x, ws=ws[:1 << 20])
    with pytest.raises(binding.Bof4Error):
        m.backward(want, ws=ws[:1 << 20])


def test_refusals():
    m = Matrix(64, 96, 0.05)
    x, r = randn((3, 96), 1), randn((3, 64), 2)
    for way in ("gemv", "gemm"):
        for bad in (dict(act="tanh"), dict(bias=r[0, :63]), dict(bias=r[0].half()), dict(mul=r[:2]), dict(mul=r.t()), dict(residual=r.half()),
                    dict(pre=r.double()), dict(out=r[:, :63]), dict(bias=r.cpu()[0]), dict(out_dtype=torch.float16)):
            with pytest.raises(ValueError):
                m.linear(way, x, **bad)
        with pytest.raises(ValueError):
            m.linear(way, x.float())
        with pytest.raises(ValueError):
            m.linear(way, x[:, :64])
        out2, r2 = _two_types((3, 64))
        with pytest.raises(binding.Bof4Error):  # over the residual with another type
            m.linear(way, x, residual=r2, out=out2)
    w = m.codes, m.scales, 64, 96, 32, m.cb, x
    p = m.packed, 64, 96, m.cb
    for call in (lambda: binding.bof4_gemv_linear(*w, None, m.k), lambda: binding.bof4_gemv_linear(*w, m.gemv_table[:-8], m.k),
                 lambda: binding.bof4_gemv_linear(*w, m.gemv_table.cpu(), m.k), lambda: binding.bof4_gemv_linear(m.codes[1:], *w[1:]),
                 lambda: binding.bof4_gemv_linear(m.codes, m.scales[1:], *w[2:]), lambda: binding.bof4_gemv_linear(m.codes.cpu(), *w[1:]),
                 lambda: binding.bof4_gemm_linear(*p, x, None, m.k), lambda: binding.bof4_gemm_linear(*p, x, m.gemm_table[:-8], m.k),
                 lambda: binding.bof4_gemm_linear(m.packed[1:], *p[1:], x), lambda: binding.bof4_gemm_linear(m.packed.cpu(), *p[1:], x),
                 lambda: binding.bof4_gemm_linear(*p, x.cpu()), lambda: binding.bof4_gemm_linear(*p, x, ws=torch.empty(1 << 24)),
                 lambda: binding.bof4_gemm_linear_backward(*p, r, m.gemm_table[:-8], m.k),
                 lambda: binding.bof4_gemm_linear_backward(m.packed[1:], *p[1:], r), lambda: binding.bof4_gemm_linear_backward(*p, r.cpu())):
        with pytest.raises(ValueError):
            call()
    for bad in (dict(act="silu"), dict(dmul=r.clone()), dict(dmul=r.clone(), mul=r), dict(dbias=r[0]), dict(dbias=torch.empty(63, device=DEV))):
        with pytest.raises((ValueError, binding.Bof4Error)):
            m.backward(r, **bad)
    with pytest.raises(ValueError):
        m.backward(r[:, :63])


def _two_types(shape):
    """A binary32 tensor, and a bfloat16 one of the same shape that begins where it does."""
    whole = torch.zeros(shape, device=DEV)
    return whole, whole.view(torch.bfloat16).reshape(-1)[:whole.numel()].view(shape)


# ------------------------------------------------------------------------------------------------ together
def test_a_gated_block_and_its_answers_forward_and_back():
    """x through a gated layer, the residual stream, the head and its log probabilities, and back to x and the bias: against
    binary64 autograd over the same decoded weights, to within the roundings of the bfloat16 tensors in between."""
    n, d, f, vocab = 160, 512, 1376, 3001
    gate, up, down, head = Matrix(f, d, 0.006), Matrix(f, d, 0.0, seed=1), Matrix(d, f, 0.006), Matrix(vocab, d, 0.006)
    x, bias = randn((n, d), 1), randn(f, 2, torch.float32, 0.1)
    target = torch.randint(-1, vocab, (n,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    bf16 = torch.bfloat16
    u = up.linear("gemm", x)
    pre = torch.empty((n, f), dtype=bf16, device=DEV)
    h = gate.linear("gemm", x, bias=bias, act="silu", mul=u, pre=pre)
    y = down.linear("gemm", h, residual=x)
    logits = head.linear("gemm", y, out_dtype=torch.float32)
    lp, entropy, _, _, stats = binding.bof4_token_logprobs(logits, target)
    g_lp, g_h = torch.full((n,), -1.0 / n, device=DEV), torch.full((n,), 0.01 / n, device=DEV)
    d_logits = binding.bof4_token_logprobs_backward(logits, stats, target, g_lp, entropy, g_h, out_dtype=bf16)
    dy = head.backward(d_logits)
    dh = down.backward(dy)
    du, dbias = torch.empty_like(u), torch.empty(f, device=DEV)
    dx = dy.float() + gate.backward(dh, act="silu", pre=pre, mul=u, dmul=du, dbias=dbias, out_dtype=torch.float32)
    dx = dx + up.backward(du, out_dtype=torch.float32)

    xr, br = x.double().requires_grad_(True), bias.double().requires_grad_(True)
    z = xr @ gate.gemm_w.t() + br
    hr = z * torch.sigmoid(z) * (xr @ up.gemm_w.t())
    logp = torch.log_softmax((hr @ down.gemm_w.t() + xr) @ head.gemm_w.t(), 1)
    has = target >= 0
    lp_r = torch.where(has, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    loss = (g_lp.double() * lp_r).sum() + (g_h.double() * -(logp.exp() * logp).sum(1)).sum()
    want_dx, want_db = torch.autograd.grad(loss, (xr, br))

    def off(a, b):
        return float((a.double() - b).norm() / b.norm())

    # seven tensors in bfloat16 (u, pre, h, y, d_logits, dy, dh and du) of half a step, 2^-9 in the mean, and dz four times:
    # under sixteen such roundings, which the activations' slopes and the softmax pass on by at most a few times
    assert off(lp, lp_r.detach()) < 16 * 2.0 ** -9 and off(dx, want_dx) < 48 * 2.0 ** -9 and off(dbias, want_db) < 48 * 2.0 ** -9


# (with results in bfloat16 these are decoded first, in workgroups of 192 rows, the columns whole or shared by 2, 4 and 8)
@pytest.mark.parametrize("rows,cols,n_tokens,share", [(500, 544, 261, 0.0), (1000, 544, 333, 0.01), (500, 1056, 390, 0.01),
                                                      (500, 2080, 261, 0.02), (500, 4128, 200, 0.01)])
def test_gemm_linear_decoded_first_for_results_in_bfloat16(rows, cols, n_tokens, share):
    m = Matrix(rows, cols, share)
    bf16, f32 = torch.bfloat16, torch.float32
    check(m, "gemm", n_tokens, "none")
    check(m, "gemm", n_tokens, "silu", mul=f32, pre=bf16)
    check(m, "gemm", n_tokens, "relu", bias=bf16, mul=bf16, residual=f32)


@pytest.mark.parametrize("way,rows,cols,n_tokens", [("gemv", 40, 96, 5), ("gemm", 40, 96, 40), ("gemm", 300, 2304, 330), ("gemm", 521, 512, 600)])
def test_row_strides_past_32_bits(way, rows, cols, n_tokens):
    """Tokens 2^32 / (n_tokens - 1) elements and more apart, forward and back, against the same call on compact tensors."""
    m = Matrix(rows, cols, 0.01)
    stride = ((1 << 32) // (n_tokens - 1) + 8 * rows + 64) // 64 * 64
    whole = torch.empty(n_tokens * stride, dtype=torch.bfloat16, device=DEV)

    def far(at, values=None):
        t = whole.as_strided((n_tokens, rows), (stride, 1), at * (rows + 3))
        return t if values is None else t.copy_(values)

    x, mul, residual = randn((n_tokens, cols), 1), randn((n_tokens, rows), 2), randn((n_tokens, rows), 3)
    pre = torch.empty((n_tokens, rows), dtype=torch.bfloat16, device=DEV)
    want = m.linear(way, x, act="silu", mul=mul, residual=residual, pre=pre)
    y, z = far(0), far(1)
    m.linear(way, x, act="silu", mul=far(2, mul), residual=far(3, residual), pre=z, out=y)
    assert torch.equal(y, want) and torch.equal(z, pre)
    if way == "gemm":
        dy, dmul = randn((n_tokens, rows), 4), torch.empty((n_tokens, rows), dtype=torch.bfloat16, device=DEV)
        dbias, dbias_far = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        dx = m.backward(dy, act="silu", pre=pre, mul=mul, dmul=dmul, dbias=dbias)
        d = far(4)
        dx_far = m.backward(far(5, dy), act="silu", pre=z, mul=far(2), dmul=d, dbias=dbias_far)
        assert torch.equal(dx_far, dx) and torch.equal(d, dmul) and torch.equal(dbias_far, dbias)


def test_most_tokens_and_columns():
    """65536 tokens of 32768 columns: x and its operands are 4 GB each.  The last tokens against binary64, forward and back."""
    m, n = Matrix(64, 32768, 0.001), 65536
    x = torch.empty((n, m.cols), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    for t in range(0, n, 4096):
        x[t:t + 4096] = torch.randn((4096, m.cols), generator=g, device=DEV, dtype=torch.bfloat16)
    y = m.linear("gemm", x)
    picked = torch.tensor([0, 1, 32767, 32768, 49151, 65503, 65504, 65535], device=DEV)
    x64, w = x[picked].double(), m.gemm_w
    want, size = x64 @ w.t().contiguous(), x64.abs() @ w.abs().t().contiguous()
    assert bool(((y[picked].double() - want).abs() <= (m.cols + 64) * U * size + 1.01 * half_step(want, torch.bfloat16)).all())
    dx = m.backward(y, out=x)  # (over x, which is done with)
    d64 = y[picked].double()
    want, size = d64 @ w, d64.abs() @ w.abs()
    assert bool(((dx[picked].double() - want).abs() <= (m.rows + 64) * U * size + 1.01 * half_step(want, torch.bfloat16)).all())


def test_refusals_of_views_that_hold_fewer_numbers_than_they_show():
    m = Matrix(64, 96, 0.05)
    x, r = randn((3, 96), 1), randn((3, 64), 2)
    wide = [torch.zeros(1, dtype=t.dtype, device=DEV).expand(2 * t.numel()) for t in (m.codes, m.scales, m.packed, m.gemm_table)]
    codes, scales, packed, table = wide
    for call in (lambda: binding.bof4_gemv_linear(codes, m.scales, 64, 96, 32, m.cb, x), lambda: binding.bof4_gemv_linear(m.codes, scales, 64, 96, 32, m.cb, x),
                 lambda: binding.bof4_gemv_linear(m.codes, m.scales.float(), 64, 96, 32, m.cb, x),
                 lambda: binding.bof4_gemv_linear(m.codes, m.scales, 64, 96, 32, m.cb, x, table, m.k),
                 lambda: binding.bof4_gemm_linear(packed, 64, 96, m.cb, x), lambda: binding.bof4_gemm_linear(m.packed, 64, 96, m.cb, x, table, m.k),
                 lambda: binding.bof4_gemm_linear_backward(packed, 64, 96, m.cb, r),
                 lambda: binding.bof4_gemm_linear(m.packed, 64, 96, m.cb, x, residual=r[:1].expand(3, 64).t().t()[:, :63])):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(residual=r[:1].expand(3, 64)), dict(mul=r[:1].expand(3, 64)), dict(out=r[:1].expand(3, 64))):
        with pytest.raises(binding.Bof4Error):  # rows on top of each other
            binding.bof4_gemm_linear(m.packed, 64, 96, m.cb, x, **kw)
    with pytest.raises(binding.Bof4Error):
        binding.bof4_gemm_linear_backward(m.packed, 64, 96, m.cb, r[:1].expand(3, 64))
    with pytest.raises(binding.Bof4Error):
        binding.bof4_token_logprobs(torch.zeros((1, 9), device=DEV).expand(3, 9))
