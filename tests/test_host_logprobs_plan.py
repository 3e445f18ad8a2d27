"""How bof4_token_logprobs cuts its rows, on the CPU: bof4_logprobs_plan.h compiled with the host's compiler."""
import ctypes
import os
import subprocess
from types import SimpleNamespace

import pytest

from test_host_gemm_plan import CSRC, HERE


def compile_plan(folder):
    so = str(folder / "logprobs_plan.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", so,
                    os.path.join(HERE, "csrc", "logprobs_plan.cpp")], check=True)
    lib = ctypes.CDLL(so)
    lib.cut.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int, ctypes.POINTER(ctypes.c_uint32)]
    lib.cut.restype = None

    def cut(n_rows, vocab, bf16):
        """Waves per workgroup, parts of a row, tiles per part, logits per tile."""
        out = (ctypes.c_uint32 * 3)()
        lib.cut(n_rows, vocab, int(bf16), out)
        return SimpleNamespace(waves=out[0], splits=out[1], tiles_per_split=out[2], tile=lib.tile_words() * (8 if bf16 else 4))

    return SimpleNamespace(cut=cut, lowest=lib.lowest, tile_word=lib.tile_word, tile_words=lib.tile_words())


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return compile_plan(tmp_path_factory.mktemp("plan"))


@pytest.mark.parametrize("per_word", [4, 8])
def test_a_lane_reads_inside_its_wave_s_tile_whatever_is_left_of_it(plan, per_word):
    n = 4 * per_word  # logits per lane; none may be left while other lanes of the wave go on
    patterns = [0, (1 << n) - 1] + [1 << i for i in range(n)] + [((1 << n) - 1) & ~((1 << i) - 1) for i in range(n)]
    for bits in patterns:
        i = plan.lowest(bits, per_word)
        assert i < n and (bits == 0 or (bits >> i & 1 and bits & ((1 << i) - 1) == 0))
        for lane in (0, 1, 31, 32, 63):
            assert plan.tile_word(bits, lane, per_word) < plan.tile_words


@pytest.mark.parametrize("bf16", [False, True])
def test_parts_hold_every_tile_and_none_is_empty(plan, bf16):
    for n in (1, 2, 3, 16, 17, 100, 511, 512, 1023, 1024, 5000):
        for vocab in (1, 7, 1023, 1024, 1025, 2048, 50257, 128000, 1 << 30):
            c = plan.cut(n, vocab, bf16)
            per_word = 8 if bf16 else 4
            tiles = -(-((vocab + 2 * per_word - 2) // per_word) // plan.tile_words)
            assert c.waves in (2, 4) and 1 <= c.splits <= 64
            assert (c.splits - 1) * c.tiles_per_split < tiles <= c.splits * c.tiles_per_split
