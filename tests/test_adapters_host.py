"""The host side of the low-rank adapters and of the gradients' norm (CPU only): refusals before anything is launched, refused launches,
the kernels that calls choose, workspaces, and what the built kernels keep in memory that should be in registers."""
import ctypes
import math
import os

import pytest

import paper_2305_08872_amd as am
from paper_2305_08872_amd import build as hip_build
from test_experts_host import which
from test_kernel_resources import _kernels

P = ctypes.c_void_p(1 << 20)      # never read
F32, BF16, FP16 = am.AMULET_FP32, am.AMULET_BF16, am.AMULET_FP16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(am.library_path()):
        hip_build.build()
    yield am.load_library()
    am.amulet_debug_fail_launches(0)


def mm(lib, type=BF16, out=BF16, tw=0, ta=0, tb=0, M=4, N=5, K=6, r=3, S=2, G=2, X=P, ldx=6, W=P, ldw=5, A=P, lda=3, ga=18, B=P, ldb=5, gb=15,
       off=P, ad=P, sc=None, T=P, ldt=3, R=P, ldr=5):
    return lib.amulet_adapters_mm(type, out, tw, ta, tb, M, N, K, r, S, G, X, ldx, W, ldw, A, lda, ga, B, ldb, gb, off, ad, sc, T, ldt, R, ldr, None)


def wgrad(lib, type=BF16, out=F32, tr=0, M=4, N=5, r=3, S=2, G=2, X=P, ldx=5, T=P, ldt=3, off=P, ad=P, R=P, ldr=3, gr=15, ws=None, n=0):
    return lib.amulet_adapters_wgrad(type, out, tr, M, N, r, S, G, X, ldx, T, ldt, off, ad, R, ldr, gr, ws, n, None)


def test_refusals_of_the_adapters(lib):
    assert mm(lib, type=F32, out=F32) == -9 and mm(lib, type=7) == -9 and mm(lib, out=FP16) == -9
    for name in ("M", "N", "K", "r", "S", "G"):
        assert mm(lib, **{name: -1}) == -2
    assert mm(lib, ad=None, S=3) == -2                          # (segments without adapters of their own: as many as adapters)
    assert mm(lib, M=2 ** 31) == -7 and mm(lib, G=2 ** 17) == -7 and mm(lib, S=2 ** 17) == -7 and mm(lib, r=2 ** 17, ldt=2 ** 17) == -7
    for name in ("X", "A", "B", "off", "T", "R"):
        assert mm(lib, **{name: None}) == -3, name
    for name, least in (("ldx", 6), ("ldw", 5), ("lda", 3), ("ldb", 5), ("ldt", 3), ("ldr", 5)):
        assert mm(lib, **{name: least - 1}) == -4, name
    assert mm(lib, tw=1, ldw=5) == -4 and mm(lib, ta=1, lda=5) == -4 and mm(lib, tb=1, ldb=2) == -4
    assert mm(lib, ga=-1) == -4 and mm(lib, gb=-1) == -4
    assert mm(lib, ldx=2 ** 24) == -7 and mm(lib, ldw=2 ** 24) == -7
    assert mm(lib, M=0, X=None, W=None, A=None, B=None, off=None, T=None, R=None) == 0
    assert mm(lib, M=2 ** 30, r=2 ** 16, ldt=2 ** 16, lda=2 ** 16) == -7       # (more workgroups than a launch holds)


def test_refusals_of_their_gradients(lib):
    assert wgrad(lib, type=F32) == -9 and wgrad(lib, out=FP16) == -9 and wgrad(lib, ad=None, S=1) == -2
    for name in ("M", "N", "r", "S", "G"):
        assert wgrad(lib, **{name: -1}) == -2
    assert wgrad(lib, M=2 ** 31) == -7 and wgrad(lib, G=2 ** 17) == -7 and wgrad(lib, r=2 ** 17) == -7
    for name in ("X", "T", "off", "R"):
        assert wgrad(lib, **{name: None}) == -3
    assert wgrad(lib, ldx=4) == -4 and wgrad(lib, ldt=2) == -4 and wgrad(lib, ldr=2) == -4 and wgrad(lib, tr=1) == -4 and wgrad(lib, gr=14) == -4
    assert wgrad(lib, ldx=16711679 // 2 + 1) == -7 and wgrad(lib, ldt=16711679 // 4 + 1) == -7
    assert wgrad(lib, ws=ctypes.c_void_p(8), n=64) == -8
    assert wgrad(lib, G=0, S=0, R=None) == 0 and wgrad(lib, N=0, R=None) == 0 and wgrad(lib, r=0, R=None) == 0
    assert wgrad(lib, G=2 ** 16, N=2 ** 20, r=64, ldx=2 ** 20, ldt=64, ldr=64, gr=2 ** 26) == -7


def arrays(types, counts, pointers):
    n = len(types)
    return n, (ctypes.c_int32 * n)(*types), (ctypes.c_int64 * n)(*counts), (ctypes.c_void_p * n)(*pointers)


def test_refusals_of_the_norm(lib):
    ok = arrays([F32, BF16], [10, 20], [1 << 20, 2 << 20])
    need = am.amulet_grad_norm_workspace_bytes(2)
    assert need == 8 * 2048 and am.amulet_grad_norm_workspace_bytes(0) == 0 and am.amulet_grad_norm_workspace_bytes(180) == need and am.amulet_grad_norm_workspace_bytes(181) == 2 * need

    def norm(a=ok, out=P, ws=P, n=need):
        return lib.amulet_grad_norm(*a, out, ws, n, None)

    def clip(a=ok, to=None, most=1.0, norm=P):
        return lib.amulet_grad_clip(*a, to, most, norm, None)

    def both(a=ok, to=None, most=1.0, out=P, ws=P, n=need):
        return lib.amulet_grad_norm_clip(*a, to, most, out, ws, n, None)
    for call in (norm, clip, both):
        assert call(arrays([F32, 3], [1, 1], [1 << 20] * 2)) == -9 and call(arrays([F32, F32], [1, -1], [1 << 20] * 2)) == -2
        assert call(arrays([F32, F32], [1, 1], [1 << 20, None])) == -3 and call((-1,) + ok[1:]) == -2 and call((2, None) + ok[2:]) == -3
        assert call(arrays([F32], [2 ** 40], [1 << 20])) == -7 and call(arrays([F32], [1], [1 << 50])) == -7
    assert norm(out=None) == -3 and norm(ws=None) == -8 and norm(n=need - 1) == -8 and norm(ws=ctypes.c_void_p(4)) == -8
    for call in (clip, both):
        assert call(most=-1.0) == -7 and call(most=math.nan) == -7
        assert call(to=(ctypes.c_void_p * 2)(1 << 20, None)) == -3
    assert clip(norm=None) == -3 and both(out=None) == -3 and both(ws=None) == -8 and both(n=need - 1) == -8
    assert lib.amulet_grad_clip(0, None, None, None, None, 1.0, None, None) == 0


def test_tensors_that_are_not_on_the_gpu_are_refused(lib):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 6, dtype=torch.bfloat16)
    a, b, t = torch.zeros(2, 6, 3, dtype=torch.bfloat16), torch.zeros(2, 3, 5, dtype=torch.bfloat16), torch.zeros(4, 3)
    off = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        am.amulet_adapters_mm(x, torch.zeros(6, 5, dtype=torch.bfloat16), a, b, off, t, torch.zeros(4, 5, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        am.amulet_adapters_wgrad(x, t, off, torch.zeros(2, 6, 3))


def test_refused_launches_come_back(lib):
    ok = arrays([F32] * 190, [10] * 190, [1 << 20] * 190)
    big = 1 << 26
    calls = [(lambda: mm(lib), 2), (lambda: wgrad(lib), 1), (lambda: mm(lib, r=0, T=None), 1), (lambda: mm(lib, N=0, R=None), 1),
             (lambda: wgrad(lib, M=20000, N=64, r=8, ldx=64, ldt=8, ldr=8, gr=512, ws=P, n=big), 2),
             (lambda: lib.amulet_grad_norm(*ok, P, P, big, None), 3), (lambda: lib.amulet_grad_norm_clip(*ok, None, 1.0, P, P, big, None), 4),
             (lambda: lib.amulet_grad_clip(*ok, None, 1.0, P, None), 2)]
    for call, launches in calls:
        am.amulet_debug_fail_launches(1)
        assert call() == -5
        am.amulet_debug_fail_launches(0)
    del launches


def test_calls_tell_which_kernel_they_ran(lib):
    def rows(M, N, K, r=16, tw=1):
        # (the first launch makes T: refused, the second is not reached, so the name is asked of a call without ranks)
        return which(lib, lambda: mm(lib, tw=tw, M=M, N=N, K=K, r=0, ldx=K, ldw=max(N, K), ldr=N, T=None))
    assert rows(16384, 4096, 4096) == ("adapters_256x256", 16384) and rows(256, 4096, 4096)[0] == "adapters_64x64_k2" and rows(8, 4096, 4096)[0] == "adapters_16x16" and rows(40, 1024, 4096)[0] == "adapters_16x32"
    assert which(lib, lambda: mm(lib, N=0, R=None)) == ("adapters_down", 4)
    assert which(lib, lambda: wgrad(lib)) == ("adapters_wgrad", 4)


def test_workspace_of_the_gradients(lib):
    """Only few and narrow matrices of many rows can use one; any size will do."""
    assert am.amulet_adapters_wgrad_workspace_bytes(64, 4096, 16, 16) == 0 and am.amulet_adapters_wgrad_workspace_bytes(0, 64, 8, 1) == 0
    assert am.amulet_adapters_wgrad_workspace_bytes(20000, 64, 8, 1) >= 2 * 64 * 8 * 4


@pytest.mark.parametrize("source", [s for s in hip_build.SOURCES if s.startswith(("adapters_down", "adapters_up", "adapters_outer", "grad_norm"))])
def test_kernels_keep_everything_in_registers(source, tmp_path):
    obj = os.path.join(hip_build.OBJ_DIR, os.path.splitext(source)[0] + ".o")
    if not os.path.exists(obj):
        hip_build.build()
    kernels = list(_kernels(obj, str(tmp_path)))
    assert len(kernels) >= 3
    assert [k for k in kernels if k[1] != 0] == []
