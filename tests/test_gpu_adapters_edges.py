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
