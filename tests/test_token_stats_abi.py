"""Host-side checks of the token-statistics and 8-bit entry points: what is refused, before any device is touched, and the
workspace sizes; and the differences of the gradient's formula in 64 bits."""
import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2603_04135_amd as P
    if not os.path.exists(P.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return P.load()


ONE = ctypes.c_void_p(256)          # never dereferenced: validation fails first


def stats(lib, shape, top_k=0, drop=(), ws_bytes=1 << 40, **other):
    from paper_2603_04135_amd.binding import HeadShape
    names = ["H", "W", "h_scale", "w_scale", "ids", "loss_pos", "logp", "lse", "entropy", "top_ids", "top_logp", "status", "ws"]
    args = {n: None if n in drop else ONE for n in names}
    args.update(other)
    return lib.dppo_token_stats(ctypes.byref(HeadShape(*shape)), top_k, *[args[n] for n in names], ws_bytes, None)


F32_ARGS = ("h_scale", "w_scale", "top_ids", "top_logp")


def test_statistics_refusals(lib):
    ok = (100, 50, 64, 1000, 1)
    assert stats(lib, (100, 50, 72, 1000, 1), drop=F32_ARGS) == 5
    assert stats(lib, (100, 50, 64, 1000, 3), drop=F32_ARGS) == 5
    assert stats(lib, (100, 101, 64, 1000, 1), drop=F32_ARGS) == 2
    assert stats(lib, (100, 50, 0, 1000, 0), drop=F32_ARGS) == 2
    assert stats(lib, (100, 50, 64, 0, 1), drop=F32_ARGS) == 2
    assert stats(lib, (100, 50, 64, 2**30 + 1, 1), drop=F32_ARGS) == 5
    assert stats(lib, (100, 0, 64, 1000, 1), drop=F32_ARGS) == 0                       # nothing to do
    for k in (-1, 65):
        assert stats(lib, ok, k, drop=("h_scale", "w_scale")) == 1
    assert stats(lib, (100, 50, 64, 10, 1), 11, drop=("h_scale", "w_scale")) == 1       # more alternatives than entries
    assert stats(lib, ok, 5, drop=("h_scale", "w_scale", "top_ids")) == 1
    assert stats(lib, ok, 0, drop=("h_scale", "w_scale")) == 1                          # top arrays without top_k
    assert stats(lib, ok, drop=F32_ARGS + ("H",)) == 1
    assert stats(lib, ok, drop=F32_ARGS + ("ids",)) == 1                                # logp without ids
    assert stats(lib, ok, drop=F32_ARGS + ("logp", "lse", "entropy")) == 1
    assert stats(lib, ok, drop=("top_ids", "top_logp")) == 1                            # scales of bfloat16 operands
    assert stats(lib, (100, 50, 128, 1000, 2), drop=F32_ARGS) == 1                      # int8 without scales
    assert stats(lib, (100, 50, 64, 1000, 2), drop=("top_ids", "top_logp")) == 5        # rows that are no multiple of 128
    assert stats(lib, (100, 50, 131072 + 128, 1000, 2), drop=("top_ids", "top_logp")) == 5
    assert stats(lib, ok, drop=F32_ARGS, H=ctypes.c_void_p(8)) == 1
    assert stats(lib, ok, drop=F32_ARGS + ("ws",)) == 4
    assert stats(lib, ok, drop=F32_ARGS, ws=ctypes.c_void_p(128)) == 4
    assert stats(lib, ok, drop=F32_ARGS, ws_bytes=1000) == 4 and b"below the minimum" in lib.dppo_last_error()


def grads(lib, shape, params=(0, 0), drop=(), ws_bytes=1 << 40, **other):
    from paper_2603_04135_amd.binding import HeadShape, StatsGradParams
    names = ["H", "W", "ids", "loss_pos", "lse", "entropy", "g_logp", "g_lse", "g_entropy", "dH", "dW", "status", "ws"]
    args = {n: None if n in drop else ONE for n in names}
    args.update(other)
    return lib.dppo_token_stats_bwd(ctypes.byref(HeadShape(*shape)), ctypes.byref(StatsGradParams(*params)),
                                    *[args[n] for n in names], ws_bytes, None)


def test_gradient_refusals(lib):
    ok = (100, 50, 64, 1000, 1)
    assert grads(lib, (100, 50, 128, 1000, 2)) == 5
    assert grads(lib, (100, 50, 72, 1000, 1)) == 5
    assert grads(lib, ok, (0, 2)) == 5
    assert grads(lib, ok, (1, 1)) == 5                                # added to in bfloat16
    assert grads(lib, (100, 50, 64, 1000, 0), (0, 1)) == 5            # bfloat16 dW of float32 operands
    for name in ("H", "W", "lse", "dH", "dW", "ids", "entropy"):
        assert grads(lib, ok, drop=(name,)) == 1, name
    assert grads(lib, ok, drop=("g_logp", "g_lse", "g_entropy")) == 1
    assert grads(lib, ok, dW=ctypes.c_void_p(264)) == 1
    assert grads(lib, ok, drop=("ws",)) == 4
    assert grads(lib, ok, ws_bytes=1 << 20) == 4


def test_8_bit_refusals(lib):
    assert lib.dppo_quantize_rows(-1, 64, 1, ONE, ONE, 128, ONE, None) == 2
    assert lib.dppo_quantize_rows(4, 0, 1, ONE, ONE, 128, ONE, None) == 2
    assert lib.dppo_quantize_rows(4, 64, 2, ONE, ONE, 128, ONE, None) == 5
    assert lib.dppo_quantize_rows(4, 129, 1, ONE, ONE, 128, ONE, None) == 2
    assert lib.dppo_quantize_rows(4, 100, 1, ONE, ONE, 100, ONE, None) == 2
    assert lib.dppo_quantize_rows(0, 64, 1, None, None, 128, None, None) == 0
    assert lib.dppo_quantize_rows(4, 64, 1, None, ONE, 128, ONE, None) == 1
    assert lib.dppo_quantize_rows(4, 64, 1, ONE, ctypes.c_void_p(8), 128, ONE, None) == 1
    assert lib.dppo_matmul_i8(4, 100, 64, ONE, ONE, ONE, ONE, ONE, 0, None) == 5
    assert lib.dppo_matmul_i8(4, 0, 128, ONE, ONE, ONE, ONE, ONE, 0, None) == 2
    assert lib.dppo_matmul_i8(-1, 100, 128, ONE, ONE, ONE, ONE, ONE, 0, None) == 2
    assert lib.dppo_matmul_i8(4, 100, 128, ONE, ONE, ONE, ONE, ONE, 2, None) == 5
    assert lib.dppo_matmul_i8(0, 100, 128, None, None, None, None, None, 0, None) == 0
    assert lib.dppo_matmul_i8(4, 100, 128, ONE, None, ONE, ONE, ONE, 0, None) == 1
    assert lib.dppo_matmul_i8(4, 100, 128, ctypes.c_void_p(8), ONE, ONE, ONE, ONE, 0, None) == 1


def test_workspace_sizes(lib):
    from paper_2603_04135_amd.binding import HeadShape

    def both(shape, k, what):
        h = ctypes.byref(HeadShape(*shape))
        return lib.dppo_token_stats_workspace_min_bytes(h, k, what), lib.dppo_token_stats_workspace_bytes(h, k, what)

    for dtype in (0, 1, 2):
        for N in (0, 1, 256, 257, 8191, 100000, 0x7fffffff):
            for D, V in ((128, 1), (128, 512), (2560, 151936), (65536, 1 << 20), (128, 1 << 30)):
                for k in (0, 1, 64):
                    if k > V:
                        continue
                    for what in (0, 1, 2):
                        least, most = both((N, N, D, V, dtype), k, what)
                        if dtype == 2 and what:
                            assert least == most == 0
                        else:
                            assert 0 < least <= most
    assert both((10, 10, 128, 100, 1), 0, 3) == (0, 0)
    assert both((10, 10, 72, 100, 1), 0, 0) == (0, 0)


def test_formula_of_the_gradient_against_differences():
    """dz = g_logp (1[y] - p) + g_lse p - g_ent p (log p + H), in 64 bits against central differences."""
    rng = np.random.default_rng(0)
    V = 12
    for _ in range(5):
        z, y = rng.normal(size=V) * 2, int(rng.integers(V))
        gl, gs, ge = rng.normal(size=3)

        def loss(z):
            lse = np.log(np.exp(z - z.max()).sum()) + z.max()
            lp = z - lse
            return gl * lp[y] + gs * lse - ge * (np.exp(lp) * lp).sum()

        lp = z - (np.log(np.exp(z - z.max()).sum()) + z.max())
        p = np.exp(lp)
        ent = -(p * lp).sum()
        dz = gl * ((np.arange(V) == y) - p) + gs * p - ge * p * (lp + ent)
        h = 1e-5
        for v in range(V):
            e = np.zeros(V)
            e[v] = h
            assert abs((loss(z + e) - loss(z - e)) / (2 * h) - dz[v]) <= 1e-8


def test_longest_int8_rows(lib):
    """Sums of D products of -128 by -128 have to stay below 2^31."""
    drop = ("top_ids", "top_logp")
    assert 128 * 128 * 130944 < 2**31 <= 128 * 128 * 131072
    assert stats(lib, (100, 50, 131072, 1000, 2), drop=drop) == 5
    assert stats(lib, (100, 50, 130944, 1000, 2), drop=drop, ws_bytes=1000) == 4           # (accepted, but for the workspace)
