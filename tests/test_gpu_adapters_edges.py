"""Low-rank adapters at the largest sizes that their calls take."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def am():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2305_08872_amd as am
    am.load_library()
    return am


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_gradients_of_as_many_rows_as_there_may_be(am):
    """2^31 - 65537 rows of one adapter: the rows and a piece's together pass 2^31."""
    M = 2 ** 31 - 65537
    X, T = torch.zeros(M, 1, dtype=BF16, device="cuda"), torch.zeros(M, 1, device="cuda")
    for row, x, t in ((0, 1.0, 3.0), (M // 2, 2.0, 5.0), (M - 1, -4.0, 0.5)):
        X[row], T[row] = x, t
    ws = torch.empty(am.amulet_adapters_wgrad_workspace_bytes(M, 1, 1, 2), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    for offsets, want in (([0, M, M], [11.0, 0.0]), ([0, 0, M], [0.0, 11.0]), ([0, M // 2 + 1, M], [13.0, -2.0])):
        R = torch.full((2, 1, 1), 7.0, device="cuda")
        am.amulet_adapters_wgrad(X, T, i32(offsets), R, ws)
        assert R.flatten().tolist() == want


@pytest.mark.parametrize("M,N,K,r", [(20_000_000, 8, 16, 128), (280_000_000, 0, 8, 4)])
def test_rows_that_a_launch_holds(am, M, N, K, r):
    """More workgroups than a grid of 16 rows to each would hold, fewer than that of the tile that is taken."""
    X = torch.randint(-2, 3, (M, K), dtype=torch.int8, device="cuda").bfloat16()
    A, B = torch.randint(-2, 3, (2, r, K), device="cuda").bfloat16(), torch.zeros(2, N, r, dtype=BF16, device="cuda")
    if N:
        B[0], B[1] = 1.0, -1.0
    T, R = torch.full((M, r), float("nan"), device="cuda"), torch.full((M, N), float("nan"), dtype=BF16, device="cuda")
    cut = M // 3 + 5
    am.amulet_adapters_mm(X, None, A, B, i32([0, cut, M - 7]), T, R, trans_a=True, trans_b=True)
    for i in range(0, M, 10_000_000):
        j = min(i + 10_000_000, M)
        want = torch.empty(j - i, r, device="cuda")
        for lo, hi, a in ((0, cut, 0), (cut, M - 7, 1), (M - 7, M, -1)):
            lo, hi = max(lo, i) - i, min(hi, j) - i
            if lo < hi:
                want[lo:hi] = X[i + lo:i + hi].float() @ A[a].float().t() if a >= 0 else 0.0
        assert torch.equal(T[i:j], want)
        if N:
            sign = torch.where(torch.arange(i, j, device="cuda")[:, None] < cut, 1.0, -1.0)
            # (whole numbers, moved by 128 stand-ins of 2^-30 of a T below 2^6 and as many roundings of sums below 2^13, then rounded to bf16)
            want = sign * want.sum(1, keepdim=True)
            assert ((R[i:j].float() - want).abs() <= 2.0 ** -8 * want.abs() + 2 * 128 * 2.0 ** -11).all()


def test_each_launch_of_a_call_can_be_refused(am):
    """The status of every launch of a call comes back, not of the first alone."""
    bf = dict(dtype=BF16, device="cuda")
    x, w, a, b = torch.zeros(40, 64, **bf), torch.zeros(96, 64, **bf), torch.zeros(2, 8, 64, **bf), torch.zeros(2, 96, 8, **bf)
    off, t, y = i32([0, 10, 40]), torch.zeros(40, 8, device="cuda"), torch.zeros(40, 96, **bf)
    wide, tall = torch.zeros(2048, 1032, **bf), torch.zeros(8200, 1032, **bf)
    wide_y, wide_t, wide_a, wide_b = torch.zeros(2048, 8200, **bf), torch.zeros(2048, 8, device="cuda"), torch.zeros(1, 8, 1032, **bf), torch.zeros(1, 8200, 8, **bf)
    long_x, long_t, d = torch.zeros(20000, 64, **bf), torch.zeros(20000, 8, device="cuda"), torch.zeros(1, 64, 8, device="cuda")
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    grads, many, norm = [torch.zeros(10, device="cuda") for _ in range(190)], [torch.zeros(9 * 8192, device="cuda") for _ in range(1000)], torch.zeros(1, device="cuda")
    kw = dict(trans_w=True, trans_a=True, trans_b=True)
    calls = [(lambda: am.amulet_adapters_mm(x, w, a, b, off, t, y, **kw), 2), (lambda: am.amulet_adapters_mm(wide, tall, wide_a, wide_b, i32([0, 2048]), wide_t, wide_y, **kw), 3),
             (lambda: am.amulet_adapters_mm(x, w, a[:, :0], b[:, :, :0], off, t[:, :0], y, **kw), 1), (lambda: am.amulet_adapters_wgrad(x, t, off, torch.empty(2, 64, 8, device="cuda")), 1),
             (lambda: am.amulet_adapters_wgrad(long_x, long_t, i32([0, 20000]), d, ws), 2), (lambda: am.amulet_grad_norm(grads, norm, ws), 3),
             (lambda: am.amulet_grad_norm_clip(grads, 1.0, norm, ws), 4), (lambda: am.amulet_grad_norm_clip(many, 1.0, norm, ws), 13), (lambda: am.amulet_grad_clip(grads, 1.0, norm), 2)]
    try:
        for n, (call, launches) in enumerate(calls):
            for k in range(1, launches + 1):
                am.amulet_debug_fail_launch(k)
                with pytest.raises(am.AmuletError) as e:
                    call()
                assert e.value.code == -5, (n, k)
            am.amulet_debug_fail_launch(launches + 1)
            call()      # (as many launches as said)
            am.amulet_debug_fail_launch(0)
    finally:
        am.amulet_debug_fail_launch(0)
    torch.cuda.synchronize()
