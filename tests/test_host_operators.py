"""CPU-only checks of the layer operators' and the log probabilities' entry points: bad arguments are refused before any GPU
call, sizes are host formulas."""
import ctypes
import os
import re
import struct

import pytest

from paper_2505_06653_amd import binding, codebooks

F32, BF16 = 0, 1


def at(address):
    return ctypes.c_void_p(address)


P = at(0x10000)


def logprobs(logits=P, kind=F32, n=4, vocab=100, ld=100, target=P, top=0, lp=P, ent=P, ids=None, top_lp=None, stats=P, ws=P,
             size=1 << 30):
    return binding.lib().bof4_token_logprobs(logits, kind, n, vocab, ld, target, top, lp, ent, ids, top_lp, stats, ws, size,
                                             None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(ws=None), dict(kind=2), dict(n=0), dict(vocab=0), dict(n=(1 << 23) + 1), dict(vocab=(1 << 30) + 1, ld=1 << 31),
    dict(ld=99), dict(target=None), dict(lp=None), dict(top=65, ids=P, top_lp=P), dict(top=1), dict(top=1, ids=P),
    dict(top=1, top_lp=P), dict(logits=at(0x10002)), dict(logits=at(0x10001), kind=BF16), dict(target=at(0x10004)),
    dict(ws=at(0x10010)), dict(ent=at(0x10002)), dict(stats=at(0x10002)), dict(top=1, ids=at(0x10004), top_lp=P)])
def test_token_logprobs_refuses(bad):
    assert logprobs(**bad) == binding.BOF4_ERR_ARG
    assert b"bof4_token_logprobs" in binding.lib().bof4_last_error()


def test_token_logprobs_workspace():
    L = binding.lib()
    assert logprobs(size=0) == binding.BOF4_ERR_WORKSPACE
    assert L.bof4_token_logprobs_workspace_bytes(0, 10, 0) == 0 and L.bof4_token_logprobs_workspace_bytes(1, 0, 0) == 0
    assert L.bof4_token_logprobs_workspace_bytes(1, 10, 65) == 0
    for n, vocab in ((1, 1), (1, 128000), (3, 1 << 30), (1000, 50257), (1 << 23, 7)):
        sizes = [L.bof4_token_logprobs_workspace_bytes(n, vocab, top) for top in (0, 1, 20, 64)]
        assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] < 1 << 24


def backward(logits=P, kind=F32, n=4, vocab=100, ld=100, stats=P, target=P, d_lp=P, ent=P, d_ent=P, out=at(0x20000), out_kind=F32,
             ld_out=100):
    return binding.lib().bof4_token_logprobs_backward(logits, kind, n, vocab, ld, stats, target, d_lp, ent, d_ent, out, out_kind,
                                                      ld_out, None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(stats=None), dict(out=None), dict(kind=7), dict(out_kind=2), dict(n=0), dict(vocab=0),
    dict(n=(1 << 23) + 1), dict(vocab=(1 << 30) + 1, ld=1 << 31, ld_out=1 << 31), dict(ld=99), dict(ld_out=99), dict(target=None),
    dict(d_lp=None), dict(ent=None), dict(d_ent=None), dict(out=P, out_kind=BF16), dict(out=P, ld_out=101),
    dict(out=at(0x20002)), dict(stats=at(0x10002)), dict(target=at(0x10004)),
    dict(n=1 << 20, vocab=1 << 20, ld=1 << 20, ld_out=1 << 20)])
def test_token_logprobs_backward_refuses(bad):
    assert backward(**bad) == binding.BOF4_ERR_ARG
    assert b"bof4_token_logprobs_backward" in binding.lib().bof4_last_error()


# ------------------------------------------------------------------------------------------------ linear layers
CB = codebooks.array(codebooks.BOF4S_MSE[64])
CBP = CB.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
BAD_CB = CB[::-1].copy()
BAD_CBP = BAD_CB.ctypes.data_as(ctypes.POINTER(ctypes.c_double))


LAYER = ("act", "bias_type", "mul_type", "residual_type", "y_type", "pre_type", "bias_dev", "mul_dev", "residual_dev", "y_dev",
         "pre_dev", "ld_mul", "ld_residual", "ld_y", "ld_pre")
GRADIENT = ("act", "dy_type", "pre_type", "mul_type", "dmul_type", "dx_type", "dy_dev", "pre_dev", "mul_dev", "dmul_dev",
            "dbias_dev", "dx_dev", "ld_dy", "ld_pre", "ld_mul", "ld_dmul", "ld_dx")


def record(packing, names, fields):
    assert set(fields) <= set(names)
    return packing.pack(*[fields.get(k) or 0 for k in names])


def layer(**kw):
    return record(binding.LAYER, LAYER, {**dict(y_dev=0x40000, y_type=BF16, ld_y=64), **kw})


def test_packed_records_are_the_header_s_structs():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bof4.h")).read()
    for name, names, packing in (("bof4_layer", LAYER, binding.LAYER), ("bof4_layer_gradient", GRADIENT, binding.LAYER_GRADIENT)):
        body = re.sub(r"/\*.*?\*/", "", text[:text.index("} " + name + ";")].rsplit("typedef struct {", 1)[1], flags=re.S)
        fields, kinds = [], ""
        for line in body.split(";"):
            if line.strip():
                words = line.replace("*", " * ").split()
                declared = [w.strip(",") for w in words if w.strip(",").endswith(("_dev", "_type")) or w.startswith("ld_") or w == "act"]
                fields += declared
                kinds += ("P" if "*" in words else "I" if "uint32_t" in words else "Q") * len(declared)
        assert tuple(fields) == names
        assert struct.Struct("@" + kinds).size == packing.size and kinds == "".join(int(n or 1) * k for n, k in re.findall(r"(\d*)([IPQ])", packing.format))


def gemv_linear(codes=P, scales=P, rows=64, cols=128, block=64, cb=CBP, table=None, k=0, x=at(0x20000), n=2, lay=None, null=False, **kw):
    return binding.lib().bof4_gemv_linear(codes, scales, rows, cols, block, cb, table, k, x, n,
                                          None if null else lay or layer(**kw), None)


def gemm_linear(packed=P, rows=64, cols=128, cb=CBP, table=None, k=0, x=at(0x20000), n=2, ws=at(0x80000), size=1 << 40, null=False, **kw):
    return binding.lib().bof4_gemm_linear(packed, rows, cols, cb, table, k, x, n, None if null else layer(**kw), ws, size, None)


BAD_LAYERS = [dict(null=True), dict(y_dev=None), dict(act=5), dict(y_type=2), dict(y_dev=0x40001), dict(ld_y=63),
              dict(bias_dev=0x50001, bias_type=BF16), dict(bias_dev=0x50002, bias_type=F32), dict(bias_dev=0x50000, bias_type=3),
              dict(mul_dev=0x50000, mul_type=BF16, ld_mul=63), dict(mul_dev=0x50000, mul_type=9, ld_mul=64),
              dict(residual_dev=0x50000, ld_residual=10), dict(residual_dev=0x50002, residual_type=F32, ld_residual=64),
              dict(pre_dev=0x50002, pre_type=F32, ld_pre=64), dict(pre_dev=0x40000, pre_type=BF16, ld_pre=64),
              dict(residual_dev=0x40000, residual_type=F32, ld_residual=64), dict(residual_dev=0x40000, residual_type=BF16, ld_residual=65),
              dict(mul_dev=0x40000, mul_type=F32, ld_mul=64), dict(bias_dev=0x40000, bias_type=BF16), dict(y_dev=0x20000)]


@pytest.mark.parametrize("bad", BAD_LAYERS + [
    dict(codes=None), dict(scales=None), dict(x=None), dict(rows=0), dict(cols=0), dict(cols=96), dict(block=48), dict(n=0),
    dict(rows=(1 << 30) + 1, ld_y=1 << 31), dict(cols=32832), dict(cb=BAD_CBP), dict(k=3), dict(k=1 << 32, table=P), dict(codes=at(0x10008)),
    dict(x=at(0x20002)), dict(scales=at(0x10001)), dict(table=at(0x10004), k=1)])
def test_gemv_linear_refuses(bad):
    assert gemv_linear(**bad) == binding.BOF4_ERR_ARG
    assert b"linear" in binding.lib().bof4_last_error()


@pytest.mark.parametrize("bad", BAD_LAYERS + [
    dict(packed=None), dict(x=None), dict(ws=None), dict(rows=0), dict(cols=0), dict(cols=100), dict(n=0), dict(n=65537),
    dict(rows=(1 << 30) + 1, ld_y=1 << 31), dict(cols=32800), dict(cb=BAD_CBP), dict(k=3), dict(k=1 << 32, table=P), dict(packed=at(0x10008)),
    dict(x=at(0x20002)), dict(ws=at(0x80010)), dict(table=at(0x10004), k=1)])
def test_gemm_linear_refuses(bad):
    assert gemm_linear(**bad) == binding.BOF4_ERR_ARG
    assert b"linear" in binding.lib().bof4_last_error()


def gemm_linear_backward(packed=P, rows=64, cols=128, cb=CBP, table=None, k=0, n=2, ws=at(0x80000), size=1 << 40, null=False, **kw):
    g = record(binding.LAYER_GRADIENT, GRADIENT,
               {**dict(dy_dev=0x20000, dy_type=BF16, ld_dy=64, dx_dev=0x40000, dx_type=BF16, ld_dx=128), **kw})
    return binding.lib().bof4_gemm_linear_backward(packed, rows, cols, cb, table, k, n, None if null else g, ws, size, None)


MUL, PRE = dict(mul_dev=0x50000, mul_type=BF16, ld_mul=64), dict(pre_dev=0x60000, pre_type=BF16, ld_pre=64)
DMUL = dict(dmul_dev=0x70000, dmul_type=BF16, ld_dmul=64)


@pytest.mark.parametrize("bad", [
    dict(null=True), dict(packed=None), dict(ws=None), dict(dy_dev=None), dict(dx_dev=None), dict(rows=0), dict(cols=0), dict(cols=100),
    dict(n=0), dict(n=65537), dict(rows=(1 << 18) + 1, ld_dy=1 << 20), dict(cols=32800, ld_dx=1 << 16), dict(cb=BAD_CBP), dict(k=3),
    dict(k=1 << 32, table=P), dict(packed=at(0x10008)), dict(ws=at(0x80010)), dict(table=at(0x10004), k=1), dict(act=5), dict(act=1),
    dict(ld_dy=63), dict(ld_dx=127), dict(dy_type=2), dict(dx_type=2), dict(dy_dev=0x20001), dict(dx_dev=0x40001), {**DMUL}, {**DMUL, **MUL},
    {**DMUL, **PRE}, {**MUL, "ld_mul": 63}, {**PRE, "ld_pre": 63}, {**MUL, **PRE, **DMUL, "ld_dmul": 63}, {**MUL, **PRE, **DMUL, "dmul_dev": 0x40000},
    {**MUL, **PRE, **DMUL, "dmul_dev": 0x20000, "dmul_type": F32}, {**MUL, **PRE, **DMUL, "dmul_dev": 0x50000, "ld_dmul": 65},
    dict(dbias_dev=0x30002), dict(dbias_dev=0x40000)])
def test_gemm_linear_backward_refuses(bad):
    assert gemm_linear_backward(**bad) == binding.BOF4_ERR_ARG
    assert b"bof4_gemm_linear_backward" in binding.lib().bof4_last_error()


@pytest.mark.parametrize("rows,cols", [(1, 32), (1001, 1504), (300, 28672), (28672, 300 // 32 * 32), (11008, 4096), (128256, 4096), (1 << 18, 32)])
def test_linear_workspaces_never_fall_as_tokens_rise_and_hold_the_product(rows, cols):
    L = binding.lib()
    for f in (L.bof4_gemm_linear_workspace_bytes, L.bof4_gemm_linear_backward_workspace_bytes):
        sizes = [f(rows, cols, n) for n in (1, 5, 31, 32, 33, 100, 128, 129, 257, 500, 1000, 2000, 3000, 9000, 65536)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    assert L.bof4_gemm_linear_workspace_bytes(rows, cols, 500) >= L.bof4_gemm_workspace_bytes(rows, cols, 500)
    assert gemm_linear(rows=rows, cols=cols, n=500, ld_y=rows, size=1000) == binding.BOF4_ERR_WORKSPACE
    assert gemm_linear_backward(rows=rows, cols=cols, n=500, ld_dy=rows, ld_dx=cols, size=1000) == binding.BOF4_ERR_WORKSPACE
    assert L.bof4_gemm_linear_workspace_bytes(0, cols, 5) == 0 and L.bof4_gemm_linear_backward_workspace_bytes(rows, cols, 0) == 0
    assert L.bof4_gemm_linear_backward_workspace_bytes((1 << 18) + 1, cols, 5) == 0
