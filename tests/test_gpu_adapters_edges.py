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
