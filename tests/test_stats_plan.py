"""Which tiles the token statistics and the 8-bit product take, from the library's own rules (host code, compiled here)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2603_04135_amd import build as B
from test_gpu_token_stats import GRADIENT_BY_A_COPY, I8_TILES

FEW, T128x96, T128x128, T256x192, T256x256 = range(5)
ROWS, COLUMNS = {T128x96: 128, T128x128: 128, T256x192: 256, T256x256: 256}, {T128x96: 96, T128x128: 128, T256x192: 192, T256x256: 256}
SOURCE = """
#include "stats_plan.h"
extern "C" int tile(int n, int V, int k2, int i8) { return dppo::logits_tile(n, V, k2, i8 != 0); }
extern "C" int eight(int n, int V, int k2) { return dppo::eight_wavefronts(n, V, k2); }
extern "C" int join_tokens(int n) { return dppo::join_tokens(n); }
extern "C" int small_grad(int N, int D, int V) { return dppo::small_grad(N, D, V); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, so = str(d / "plan.cpp"), str(d / "plan.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-shared", "-fPIC", "-I", B.CSRC, src, "-o", so], check=True)
    return ctypes.CDLL(so)


def test_launches_stay_below_2_to_the_32_threads(plan):
    """The runtime launches the number of threads modulo 2^32. Chunks have at most 2^31 logits, and 256 tokens in any case."""
    for V in (2 ** 30, 2 ** 30 - 1, 2 ** 30 - 128, 2 ** 29, 2 ** 27 + 1, 2 ** 23, 2 ** 20 + 1, 151936, 1000):
        for n in (17, 64, 96, 97, 100, 128, 129, 192, 193, 255, 256, max(256, min(32768, 2 ** 31 // V))):
            for k2 in (64, 128, 512, 576, 4096):
                for i8 in (0, 1):
                    t = plan.tile(n, V, k2, i8)
                    threads = 256 if t == T128x96 or t == T128x128 and not plan.eight(n, V, k2) else 512
                    assert -(-V // ROWS[t]) * -(-n // COLUMNS[t]) * threads < 2 ** 32, (n, V, k2, t)


def test_gpu_tests_reach_the_tiles_they_are_meant_for(plan):
    for name, n, D, V in I8_TILES:
        assert plan.tile(n, V, D // 2, 1) == {"256x256": T256x256, "256x192": T256x192}[name]
        assert n % COLUMNS[plan.tile(n, V, D // 2, 1)] and V % 256
    for N, D, V in GRADIENT_BY_A_COPY:
        assert N > 4096 + D and not plan.small_grad(N, D, V)


def test_tokens_of_a_join(plan):
    """Both sides of each line (see join_tokens for what was measured there)."""
    for n, tokens in ((1, 1), (256, 1), (257, 4), (512, 4), (513, 8), (1000, 8), (2048, 8), (2049, 16), (8191, 16)):
        assert plan.join_tokens(n) == tokens
