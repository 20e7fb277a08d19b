"""The mixture-of-experts operators' host side (CPU only): refusals before anything is launched, launches that are refused,
the kernels that calls choose, and what the built kernels keep in memory that should be in registers."""
import ctypes
import os

import pytest

import paper_2305_08872_amd as am
from paper_2305_08872_amd import build as hip_build
from test_kernel_resources import _kernels

P = ctypes.c_void_p(1 << 20)      # never read
F32, BF16, FP16 = am.AMULET_FP32, am.AMULET_BF16, am.AMULET_FP16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(am.library_path()):
        hip_build.build()
    yield am.load_library()
    am.amulet_debug_fail_launches(0)


def grouped(lib, type=BF16, out=BF16, tb=0, M=4, N=5, K=6, G=2, A=P, lda=6, rows=None, a_rows=4, B=P, ldb=5, gb=30, off=P, R=P, ldr=5):
    return lib.amulet_grouped_mm(type, out, tb, M, N, K, G, A, lda, rows, a_rows, B, ldb, gb, off, R, ldr, None)


def test_refusals_of_the_products(lib):
    assert grouped(lib, type=F32, out=F32) == -9 and grouped(lib, type=7) == -9 and grouped(lib, out=FP16) == -9
    for name in ("M", "N", "K", "G", "a_rows"):
        assert grouped(lib, **{name: -1}) == -2
    assert grouped(lib, M=2 ** 31) == -7 and grouped(lib, G=2 ** 17) == -7
    for name in ("A", "B", "off", "R"):
        assert grouped(lib, **{name: None}) == -3
    assert grouped(lib, lda=5) == -4 and grouped(lib, ldb=4) == -4 and grouped(lib, ldr=4) == -4 and grouped(lib, tb=1, ldb=5) == -4 and grouped(lib, gb=-1) == -4
    assert grouped(lib, lda=2 ** 24) == -7 and grouped(lib, ldb=2 ** 24) == -7
    assert grouped(lib, M=0, A=None, B=None, off=None, R=None) == 0 and grouped(lib, N=0, R=None) == 0
    assert am.amulet_strerror(-9).startswith("unknown element type")

    def wgrad(type=BF16, out=F32, tr=0, M=4, N=5, K=6, G=2, A=P, lda=6, rows=None, a_rows=4, D=P, ldd=5, off=P, R=P, ldr=5, gr=30, ws=None, n=0):
        return lib.amulet_grouped_mm_wgrad(type, out, tr, M, N, K, G, A, lda, rows, a_rows, D, ldd, off, R, ldr, gr, ws, n, None)
    assert wgrad(type=F32) == -9 and wgrad(out=FP16) == -9 and wgrad(K=-1) == -2 and wgrad(M=2 ** 31) == -7
    for name in ("A", "D", "off", "R"):
        assert wgrad(**{name: None}) == -3
    assert wgrad(lda=5) == -4 and wgrad(ldd=4) == -4 and wgrad(ldr=4) == -4 and wgrad(tr=1) == -4 and wgrad(gr=29) == -4
    assert wgrad(ws=ctypes.c_void_p(8), n=64) == -8 and wgrad(lda=2 ** 24) == -7
    assert wgrad(G=0, R=None) == 0 and wgrad(N=0, R=None) == 0

    def fp8(out=BF16, tb=0, M=4, N=5, K=300, G=2, A=P, lda=300, sa=P, lsa=4, rows=None, a_rows=4, B=P, ldb=5, gb=1500, sb=P, lsb=1, gsb=3, off=P, R=P, ldr=5):
        return lib.amulet_grouped_mm_fp8(out, tb, M, N, K, G, A, lda, sa, lsa, rows, a_rows, B, ldb, gb, sb, lsb, gsb, off, R, ldr, None)
    assert fp8(out=3) == -9 and fp8(K=-1) == -2 and fp8(sa=None) == -3 and fp8(sb=None) == -3 and fp8(lsa=3) == -4
    assert fp8(tb=1, ldb=300) == -4 and fp8(rows=P, a_rows=9) == -4 and fp8(gsb=-1) == -4
    assert lib.amulet_mm_fp8(BF16, 0, 4, 5, 300, P, 300, P, 4, P, 5, P, 0, P, 5, None) == -4


def test_refusals_of_the_router_the_combine_and_the_quantiser(lib):
    def route(type=F32, T=100, E=8, k=2, X=P, ldx=8, e=P, w=P, p=P, t=P, o=P, ws=P, n=1 << 20):
        return lib.amulet_route(type, T, E, k, X, ldx, 1, e, w, p, t, o, ws, n, None)
    assert route(type=3) == -9 and route(T=-1) == -2 and route(k=0) == -2 and route(k=9) == -2 and route(E=0) == -2
    assert route(E=1025, ldx=1025) == -7 and route(E=100, k=65, ldx=100) == -7 and route(ldx=7) == -4
    for name in ("X", "e", "w", "p", "t", "o"):
        assert route(**{name: None}) == -3
    need = am.amulet_route_workspace_bytes(100, 8)
    assert need == 2 * 8 * 4 and am.amulet_route_workspace_bytes(64, 8) == 0 and am.amulet_route_workspace_bytes(10 ** 6, 1024) <= 256 * 1024 * 4
    assert route(ws=None) == -8 and route(n=need - 1) == -8 and route(ws=ctypes.c_void_p(2)) == -8
    g = lib.amulet_route_grad
    assert g(F32, 4, 8, 2, None, 8, 0, P, P, P, P, 8, None) == -3 and g(F32, 4, 8, 2, None, 8, 1, P, P, P, P, 7, None) == -4 and g(F32, 0, 8, 2, None, 8, 1, None, None, None, None, 8, None) == 0
    c = lib.amulet_combine
    assert c(5, 4, 2, 8, 8, P, 8, P, P, P, 8, None) == -9 and c(F32, 4, -2, 8, 8, P, 8, P, P, P, 8, None) == -2 and c(F32, 4, 2, 8, 8, None, 8, P, P, P, 8, None) == -3
    assert c(F32, 4, 2, 8, 8, P, 7, P, P, P, 8, None) == -4 and c(F32, 4, 2, 8, 8, P, 8, P, P, P, 7, None) == -4 and c(F32, 2 ** 30, 8, 8, 8, P, 8, P, P, P, 8, None) == -7
    assert c(F32, 0, 2, 8, 8, None, 8, None, None, None, 8, None) == 0
    d = lib.amulet_combine_grad
    assert d(F32, 4, 2, 8, 8, None, 8, P, P, P, 8, P, 8, P, None) == -3 and d(F32, 4, 2, 8, 8, P, 8, P, P, P, 8, P, 7, P, None) == -4 and d(F32, 4, 2, -8, 8, P, 8, P, P, P, 8, P, 8, P, None) == -2
    q = lib.amulet_quantize_fp8
    assert q(3, 4, 200, P, 200, P, 200, P, 4, None) == -9 and q(F32, 4, 200, P, 199, P, 200, P, 4, None) == -4 and q(F32, 4, 200, P, 200, P, 200, P, 3, None) == -4
    assert q(F32, 4, 200, None, 200, P, 200, P, 4, None) == -3 and q(F32, -4, 200, P, 200, P, 200, P, 4, None) == -2 and q(F32, 0, 200, None, 200, None, 200, None, 4, None) == 0
    b = lib.amulet_quantize_fp8_blocks
    assert b(F32, 2, 4, 200, P, 200, 800, P, 200, 800, P, 1, 2, None) == -4 and b(F32, 2, 4, 200, P, 200, 800, P, 200, 799, P, 2, 2, None) == -4
    assert b(F32, 2, 4, 200, P, 200, 800, P, 200, 800, None, 2, 2, None) == -3


def test_refused_launches_come_back(lib):
    for call in (lambda: lib.amulet_route(F32, 1000, 8, 2, P, 8, 1, P, P, P, P, P, P, 1 << 20, None),
                 lambda: lib.amulet_grouped_mm_wgrad(BF16, F32, 0, 20000, 64, 64, 1, P, 64, None, 20000, P, 64, P, P, 64, 4096, P, 1 << 26, None),
                 lambda: grouped(lib), lambda: lib.amulet_route(F32, 8, 8, 2, P, 8, 1, P, P, P, P, P, None, 0, None),
                 lambda: lib.amulet_combine(F32, 4, 2, 8, 8, P, 8, P, P, P, 8, None), lambda: lib.amulet_quantize_fp8(BF16, 4, 200, P, 200, P, 200, P, 4, None),
                 lambda: lib.amulet_mm_fp8(BF16, 0, 4, 5, 300, P, 300, P, 4, P, 5, P, 3, P, 5, None)):
        am.amulet_debug_fail_launches(1)
        assert call() == -5
    am.amulet_debug_fail_launches(0)


def which(lib, call):
    am.amulet_debug_fail_launches(1)
    try:
        assert call() == -5
    finally:
        am.amulet_debug_fail_launches(0)
    name, word, rows = am.amulet_recent_kernel().split()
    assert word == "rows"
    return name, int(rows)


def test_calls_tell_which_kernel_they_ran(lib):
    def rows(M, N, K, G, tb=1):
        return which(lib, lambda: grouped(lib, tb=tb, M=M, N=N, K=K, G=G, lda=K, a_rows=M, ldb=max(N, K), gb=N * K, ldr=N))
    assert rows(32768, 4096, 4096, 32) == ("grouped_mm_256x256", 32768)
    assert rows(8192, 1024, 1024, 8)[0] == "grouped_mm_128x128" and rows(256, 4096, 4096, 1)[0] == "grouped_mm_64x64_k2"
    assert rows(48, 2048, 2048, 64)[0] == "grouped_mm_16x32" and rows(64, 512, 4096, 1)[0] == "grouped_mm_16x32"
    # a gather from rows that lie more than 4 GiB apart: not the tile whose offsets have 32 bits
    far = which(lib, lambda: grouped(lib, tb=1, M=32768, N=4096, K=4096, G=32, lda=4096, rows=P, a_rows=10 ** 6, ldb=4096, gb=1 << 24, ldr=4096))
    assert far[0] == "grouped_mm_128x128"
    fp8 = lambda out: which(lib, lambda: lib.amulet_mm_fp8(out, 1, 8192, 8192, 4096, P, 4096, P, 8192, P, 4096, P, 32, P, 8192, None))[0]   # noqa: E731
    assert fp8(BF16) == "mm_fp8_256x256" and fp8(F32) == "mm_fp8_128x128"       # (8-bit products with 32-bit results: no such tile)
    assert which(lib, lambda: lib.amulet_route(F32, 1000, 8, 2, P, 8, 1, P, P, P, P, P, P, 1 << 20, None)) == ("route", 1000)
    assert which(lib, lambda: lib.amulet_combine_grad(F32, 4, 2, 8, 8, P, 8, P, P, P, 8, P, 8, P, None)) == ("combine_grad", 4)


def test_workspace_of_the_gradients(lib):
    """Only sums over many rows that few outputs have can use one; any size will do."""
    assert am.amulet_grouped_mm_wgrad_workspace_bytes(64, 2048, 2048, 16) == 0
    assert am.amulet_grouped_mm_wgrad_workspace_bytes(20000, 64, 64, 1) >= 2 * 64 * 64 * 4
    assert am.amulet_grouped_mm_wgrad_workspace_bytes(0, 64, 64, 1) == 0


@pytest.mark.parametrize("source", [s for s in hip_build.SOURCES if s.startswith(("experts_mm", "experts_sums", "route", "combine", "quantize"))])
def test_kernels_keep_everything_in_registers(source, tmp_path):
    obj = os.path.join(hip_build.OBJ_DIR, os.path.splitext(source)[0] + ".o")
    if not os.path.exists(obj):
        hip_build.build()
    kernels = list(_kernels(obj, str(tmp_path)))
    assert len(kernels) >= 4
    assert [k for k in kernels if k[1] != 0] == []
