"""The host's rules of bof4_gemm_linear (which kernel takes a layer and the workspace that follows), on the CPU: bof4_gemm_plan.h
compiled with the host's compiler."""
import ctypes
import os
import subprocess

import pytest

from paper_2505_06653_amd import binding
from test_host_gemm_plan import ANY_SIZE, CSRC, DECODED, HERE, NARROW, rules, shapes  # noqa: F401 (rules: a fixture)


class LayerPlan(ctypes.Structure):
    _fields_ = [(k, ctypes.c_uint32) for k in ("way", "decoded_split", "decoded_slab_tiles", "flush", "carry")] + [
        (k, ctypes.c_uint64) for k in ("need", "slab_bytes")]


@pytest.fixture(scope="module")
def layers(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "layer_plan.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", so,
                    os.path.join(HERE, "csrc", "layer_plan.cpp")], check=True)
    lib = ctypes.CDLL(so)
    lib.layer_plan.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_int, ctypes.c_uint64,
                               ctypes.POINTER(LayerPlan)]
    lib.layer_plan.restype = None
    lib.layer_workspace_bytes.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32]
    lib.layer_workspace_bytes.restype = ctypes.c_uint64

    def plan(rows, cols, n_tokens, listed, bf16, ws_bytes=ANY_SIZE):
        p = LayerPlan()
        lib.layer_plan(rows, cols, n_tokens, int(listed), int(bf16), ws_bytes, ctypes.byref(p))
        return p

    plan.workspace_bytes = lib.layer_workspace_bytes
    return plan


def test_layer_workspace_bytes_is_enough_for_both_types_of_results(layers):
    n_decoded = [0, 0]
    for rows, cols, n in shapes(3000, 5):
        own = layers.workspace_bytes(rows, cols, n)
        for bf16 in (False, True):
            for listed in (False, True):
                best = layers(rows, cols, n, listed, bf16)
                assert layers(rows, cols, n, listed, bf16, own).way == best.way, (rows, cols, n, listed, bf16)
                assert layers(rows, cols, n, listed, bf16, best.need - 1).way < best.way or best.way == NARROW
                assert best.way != DECODED or best.slab_bytes <= 256 << 20
                n_decoded[bf16] += best.way == DECODED
    assert n_decoded[1] > n_decoded[0] > 500
    for rows, cols, n in shapes(100, 6):
        assert binding.bof4_gemm_linear_workspace_bytes(rows, cols, n) == layers.workspace_bytes(rows, cols, n)
        sizes = [layers.workspace_bytes(rows, cols, m) for m in range(1, n, 13)] + [layers.workspace_bytes(rows, cols, n)]
        assert sizes == sorted(sizes)


def test_layer_with_binary32_results_keeps_the_products_way(layers, rules):  # noqa: F811
    for rows, cols, n in shapes(300, 7):
        for listed in (False, True):
            a, b = layers(rows, cols, n, listed, False), rules(rows, cols, n, listed)
            assert (a.way, a.decoded_split, a.decoded_slab_tiles, a.flush, a.carry) == (
                b.way, b.decoded_split, b.decoded_slab_tiles, b.flush, b.carry)


def test_layer_with_bfloat16_results_is_decoded_first_from_fewer_tokens(layers):
    for bf16, way in ((False, False), (True, True)):
        assert (layers(11008, 4096, 300, False, bf16).way == DECODED) == way
    assert layers(4096, 11008, 300, False, True).way != DECODED  # 59 us against 69
