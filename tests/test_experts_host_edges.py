"""The mixture-of-experts operators' host side at the edges of their ranges (CPU only): what a call with two launches tells of them."""
import ctypes
import os

import pytest

import paper_2305_08872_amd as am
from paper_2305_08872_amd import build as hip_build

P = ctypes.c_void_p(1 << 20)      # never read
F32, BF16, FP16 = am.AMULET_FP32, am.AMULET_BF16, am.AMULET_FP16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(am.library_path()):
        hip_build.build()
    yield am.load_library()
    am.amulet_debug_fail_launches(0)


def note(call, status=-5):
    """amulet_recent_kernel after a call whose launch is refused, as (name, fields)."""
    am.amulet_debug_fail_launches(1)
    try:
        assert call() == status
    finally:
        am.amulet_debug_fail_launches(0)
    words = am.amulet_recent_kernel().split()
    return words[0], dict(zip(words[1::2], map(int, words[2::2])))


def test_a_call_tells_of_its_second_launch(lib):
    def rows(M, N, K, G):
        return note(lambda: lib.amulet_grouped_mm(BF16, BF16, 1, M, N, K, G, P, K, None, M, P, K, N * K, P, P, N, None))
    assert rows(4096, 4500, 1203, 1) == ("grouped_mm_256x256", {"rows": 4096, "last_columns": 128})
    assert rows(4096, 4096, 1203, 1) == ("grouped_mm_256x256", {"rows": 4096})        # whole rounds
    assert rows(4114, 4501, 1211, 2) == ("grouped_mm_256x256", {"rows": 4114, "last_columns": 128})

    def fp8(N):
        return note(lambda: lib.amulet_mm_fp8(BF16, 1, 4096, N, 2111, P, 2111, P, 4096, P, 2111, P, 17, P, N, None))
    assert fp8(4501) == ("mm_fp8_256x256", {"rows": 4096, "last_columns": 128})
    assert fp8(4096) == ("mm_fp8_256x256", {"rows": 4096})

    def sums(M, N, K, G, ws, n):
        return note(lambda: lib.amulet_grouped_mm_wgrad(BF16, F32, 0, M, N, K, G, P, K, None, M, P, N, P, P, N, N * K, ws, n, None))
    assert sums(20000, 64, 64, 1, None, 0) == ("grouped_mm_wgrad_64x64", {"rows": 20000})
    name, told = sums(20000, 64, 64, 1, P, 1 << 26)
    assert name == "grouped_mm_wgrad_64x64" and told["parts"] > 1
    # a call of the products after it has none
    assert rows(4096, 4096, 1203, 1)[1] == {"rows": 4096}


def test_written_matrices_at_any_distance_that_keeps_them_apart(lib):
    def wgrad(K, N, G, ldr, gr, tr=0):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_grouped_mm_wgrad(BF16, F32, tr, 4, N, K, G, P, K, None, 4, P, N, P, P, ldr, gr, None, 0, None)
    assert wgrad(6, 5, 3, 8, 45) == -5 and wgrad(6, 5, 3, 8, 44) == -4             # the last row without its padding
    assert wgrad(6, 5, 3, 15, 5) == -5 and wgrad(6, 5, 3, 14, 5) == -4 and wgrad(6, 5, 3, 15, 4) == -4   # rows in turn
    assert wgrad(6, 5, 3, 6, 30, tr=1) == -5 and wgrad(6, 5, 3, 6, 29, tr=1) == -4
    assert wgrad(1, 5, 3, 5, 5) == -5 and wgrad(1, 5, 3, 5, 0) == -4 and wgrad(6, 5, 3, 8, -45) == -4
    assert wgrad(6, 5, 2, 2 ** 62, 5) == -5 and wgrad(6, 5, 2, 2 ** 62, 2 ** 62) == -4 and wgrad(6, 5, 1, 5, 0) == -5

    def blocks(G, M, K, ldq, gq, lds, gs):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_quantize_fp8_blocks(F32, G, M, K, P, K, M * K, P, ldq, gq, P, lds, gs, None)
    assert blocks(2, 4, 200, 208, 824, 2, 2) == -5 and blocks(2, 4, 200, 208, 823, 2, 2) == -4
    assert blocks(2, 4, 200, 400, 200, 2, 2) == -5 and blocks(2, 300, 200, 200, 60000, 3, 8) == -5 and blocks(2, 300, 200, 200, 60000, 3, 7) == -4
    assert blocks(2, 300, 200, 200, 60000, 4, 2) == -5 and blocks(2, 300, 200, 200, 60000, 3, 2) == -4
    am.amulet_debug_fail_launches(0)


def test_the_longest_pitch_is_one_of_bytes(lib):
    most = 16711679

    def mm16(lda=64, ldb=64):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_grouped_mm(BF16, F32, 1, 4, 5, 64, 1, P, lda, None, 4, P, ldb, 0, P, P, 5, None)

    def mm8(lda=64, ldb=64):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_mm_fp8(BF16, 1, 4, 5, 64, P, lda, P, 4, P, ldb, P, 1, P, 5, None)
    assert mm8(lda=most) == mm8(ldb=most) == -5 and mm8(lda=most + 1) == mm8(ldb=most + 1) == -7
    assert mm16(lda=most // 2) == mm16(ldb=most // 2) == -5 and mm16(lda=most // 2 + 1) == mm16(ldb=most // 2 + 1) == -7
    am.amulet_debug_fail_launches(0)


def test_large_results_of_the_gradients_are_taken(lib):
    """128 matrices of 8192 x 8192 (17 GB of bf16): only a launch that adds up ranges has a limit on R's tiles of its own."""
    assert note(lambda: lib.amulet_grouped_mm_wgrad(BF16, BF16, 0, 65536, 8192, 8192, 128, P, 8192, None, 65536, P, 8192, P, P, 8192, 8192 * 8192, None, 0, None)) \
        == ("grouped_mm_wgrad_256x256", {"rows": 65536})
    assert note(lambda: lib.amulet_grouped_mm_wgrad(BF16, BF16, 0, 300, 8192, 8192, 128, P, 8192, None, 300, P, 8192, P, P, 8192, 8192 * 8192, P, 1 << 34, None))[1] \
        == {"rows": 300}


def test_limits_of_the_small_kernels_are_those_of_their_launches(lib):
    """What a launch can hold is taken; what it cannot is refused by its size, not by the launch."""
    def q(M, K):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_quantize_fp8(BF16, M, K, P, K, P, K, P, M, None)
    assert q(1 << 20, 1 << 14) == -5 and q(1 << 22, 1 << 14) == -5          # 16 rows x 512 columns to a workgroup of 256
    assert q(1 << 23, 1 << 14) == -7

    def combine(type, T, k, H):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_combine(type, T, k, H, 100, P, H, None, P, P, H, None)

    def combine_grad(T, k, H):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_combine_grad(BF16, T, k, H, 100, P, H, None, P, P, H, P, H, None, None)
    assert combine(BF16, (1 << 24) - 4, 4, 2048) == -5 and combine(BF16, 1 << 24, 4, 2049) == -7     # four waves of 512 columns
    assert combine(F32, (1 << 24) - 4, 4, 1024) == -5 and combine(F32, 1 << 24, 4, 1025) == -7       # ... of 256
    assert combine(BF16, (1 << 24) - 4, 100, 512) == -5 and combine_grad((1 << 26) - 4, 1, 9000) == -5 and combine_grad(1 << 24, 4, 64) == -7

    def route_grad(T, E, k):
        am.amulet_debug_fail_launches(1)
        return lib.amulet_route_grad(F32, T, E, k, None, E, 1, P, P, P, P, E, None)
    assert route_grad((1 << 28) - 16, 8, 2) == -5 and route_grad(1 << 28, 8, 2) == -7          # 16 tokens to a workgroup
    assert route_grad((1 << 26) - 4, 300, 2) == -5 and route_grad(1 << 26, 300, 2) == -7       # ... 4
    am.amulet_debug_fail_launches(0)


def test_a_refused_workspace_is_named_as_one(lib):
    """The router's counts and the sums of ranges lie in a workspace too, not only packed copies."""
    text = am.amulet_strerror(-8)
    assert "workspace" in text and "packed" not in text and "aligned" in text


def test_sizes_whose_tiles_pass_64_bits(lib):
    """2^64 tiles of 64 x 64: refused or without a workspace, in a process of its own (the number was a divisor once)."""
    code = """
import ctypes, paper_2305_08872_amd as am
lib, P = am.load_library(), ctypes.c_void_p(1 << 20)
n = 1 << 30
assert am.amulet_grouped_mm_wgrad_workspace_bytes(1, n, n, 65536) == 0
assert am.amulet_grouped_mm_wgrad_workspace_bytes(1 << 30, n, n, 32768) == 0
assert lib.amulet_grouped_mm_wgrad(1, 0, 0, 0, n, n, 65536, P, n, None, 0, P, n, P, P, n, n * n, P, 1 << 30, None) == -7
assert lib.amulet_grouped_mm_wgrad(1, 0, 0, 0, 2147418111, 2147418111, 65536, P, n, None, 0, P, n, P, P, 2147418111, 2147418111 ** 2, None, 0, None) == -7
"""
    import subprocess
    import sys
    res = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, (res.returncode, res.stderr[-2000:])


def test_a_tile_that_the_launch_holds_is_taken(lib):
    """Sizes whose fastest tile by the estimate would need more workgroups than a launch holds: the fastest of the others."""
    def fp8(out, M, N, K, G):
        blocks = (N + 127) // 128
        return note(lambda: lib.amulet_grouped_mm_fp8(out, 0, M, N, K, G, P, K, P, M, None, M, P, N, N * K, P, blocks, blocks * ((K + 127) // 128), P, P, N, None))
    for out in (F32, BF16):
        assert fp8(out, 17018, 264383, 65, 1801)[0].startswith("mm_fp8_") and fp8(out, 565, 1038212, 71, 584)[1] == {"rows": 565}
    assert note(lambda: lib.amulet_grouped_mm(BF16, BF16, 0, 17018, 264383, 65, 1801, P, 65, None, 17018, P, 264383, 264383 * 65, P, P, 264383, None))[1] == {"rows": 17018}
    am.amulet_debug_fail_launches(1)
    n = 1 << 30                                              # more than any tile's
    assert lib.amulet_grouped_mm(BF16, BF16, 0, n, n, 1, 1, P, 1, None, n, P, 1, 0, P, P, n, None) in (-4, -7)
    assert lib.amulet_grouped_mm(BF16, BF16, 1, n, n, 1, 1, P, 1, None, n, P, 1, 0, P, P, n, None) == -7
    am.amulet_debug_fail_launches(0)
