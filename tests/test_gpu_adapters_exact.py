"""Low-rank adapters and their matrices' gradients on sums of whole numbers (test_adapters_exact_host.py says what they show and what they may be off
by): every tile of both products, both ways of adding the adapters, ranks and segments that take several passes, rows that several waves and pieces share."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_adapters_exact_host import LIMIT, fine_limit, fine_problem, mm_answer, mm_problem, outer_answer, outer_problem  # noqa: E402

F32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
ALONG, ACROSS = (True, True, True), (False, False, False)


@pytest.fixture(scope="module")
def am():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2305_08872_amd as am
    am.load_library()
    return am


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run_mm(am, seed, sizes, which, G, N, K, r, dtype, out, trans, spare=0, wide=False):
    X, W, A, B, scales, at, who = mm_problem(seed, sizes, which, G, N, K, r, trans, spare, wide)
    X, W, A, B = (v.cuda().to(dtype) for v in (X, W, A, B))
    T, R = torch.full((X.shape[0], r), float("nan"), device="cuda"), torch.full((X.shape[0], N), float("nan"), dtype=out, device="cuda")
    am.amulet_adapters_mm(X, W, A, B, i32(at), T, R, adapters=None if which is None else i32(which), scales=scales.cuda(), trans_w=trans[0], trans_a=trans[1], trans_b=trans[2])
    name = am.amulet_recent_kernel().split()[0]
    wantT, wantR = mm_answer(X, W, A, B, scales, at, who, trans)
    assert torch.equal(T.double(), wantT), name
    return name, R.double(), wantR


MM = [
    # rows of few segments: the second product's tiles, ranks of one and two passes
    ("16x16", [1] * 8, None, 8, 4096, 4096, 16), ("16x32", [3, 30, 0, 7], [1, -1, 0, 1], 2, 1024, 4096, 33), ("64x64_k2", [150, 106], None, 2, 4096, 4096, 16),
    ("64x64", [40, 0, 90, 70], [0, 2, 1, 0], 3, 520, 264, 20), ("64x64", [400, 500], None, 2, 520, 136, 100),
    ("64x128", [300, 30, 670], [1, -1, 0], 2, 4104, 520, 72), ("64x128", [1000], None, 1, 4104, 520, 128),
    ("128x128", [700, 1300], [1, 0], 2, 4104, 136, 72), ("128x128", [2000], None, 1, 4104, 136, 128), ("128x128", [333, 0, 1667], None, 3, 4104, 264, 16),
    ("256x256", [900, 1100], None, 2, 8200, 1032, 64), ("256x256", [1999], None, 1, 8200, 1032, 72), ("256x256", [500, 1, 1500], [1, 0, 1], 2, 8200, 1032, 128),
]


@pytest.mark.parametrize("trans", [ALONG, ACROSS])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (FP16, FP16), (FP16, F32)])
@pytest.mark.parametrize("tile,sizes,which,G,N,K,r", MM)
def test_all_of_t_enters(am, tile, sizes, which, G, N, K, r, dtype, out, trans):
    print("exact", tile, sizes[:8], N, K, r, dtype, out, trans, flush=True)
    name, R, want = run_mm(am, K + r, sizes, which, G, N, K, r, dtype, out, trans)
    assert name == ("adapters_64x64" if tile == "64x64_k2" and trans == ACROSS else "adapters_" + tile)
    off = (R - want).abs()
    assert float(off.max()) <= LIMIT, (name, int((off > LIMIT).sum()))


@pytest.mark.parametrize("trans", [ALONG, ACROSS])
@pytest.mark.parametrize("tile,sizes,which,G,N,K,r", [("16x16", [1] * 8, None, 8, 4096, 64, 16), ("64x64", [40, 0, 90, 70], [0, 2, 1, 0], 3, 520, 64, 20), ("64x128", [300, 700], None, 2, 4104, 520, 72),
                                                      ("128x128", [700, 1300], None, 2, 4104, 136, 64), ("256x256", [900, 1100], None, 2, 8200, 1032, 72)])
def test_all_of_an_fp16_b_enters(am, tile, sizes, which, G, N, K, r, trans):
    """T of 10 bits, B of 11, sums below 2^22, whose step is 2^-1 at most; a piece of T, of which up to two are stand-ins, times two of B, of two ranks: 8 steps."""
    print("exact b", tile, sizes[:8], N, K, r, trans, flush=True)
    name, R, want = run_mm(am, K + r, sizes, which, G, N, K, r, FP16, F32, trans, wide=True)
    assert name in ("adapters_" + tile, "adapters_64x64")
    assert float((R - want).abs().max()) <= 4.0


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("trans", [ALONG, ACROSS])
@pytest.mark.parametrize("sizes,K,r", [([1500, 0, 400], 1032, 16), ([4000, 5000], 1032, 16), ([16000, 3000], 1040, 16), ([16000, 3000], 1040, 12), ([17, 3, 0, 2] * 200, 1032, 16),
                                       ([2000, 3000], 2056, 32), ([4000, 5000], 1032, 32), ([16000, 3000], 1040, 32), ([16000, 3000], 1040, 20), ([17, 3, 0, 2] * 200, 1032, 24),
                                       ([2000, 3000], 1032, 64), ([4000, 5000], 1032, 64), ([4000, 5000], 1032, 100), ([17, 3, 0, 2] * 200, 1032, 40), ([300], 4104, 128)])
def test_the_first_product(am, sizes, K, r, trans, dtype):
    """Its tiles go by rows, segments and rank: 16, 32 or 64 rows, of 16, 32 or 64 ranks; rings that go round several times."""
    print("first product", len(sizes), sizes[:4], K, r, trans, dtype, flush=True)
    G = len(sizes)
    X, W, A, B, scales, at, who = mm_problem(r, sizes, None, G, 8, K, r, trans, spare=3)
    X, A = X.cuda().to(dtype), A.cuda().to(dtype)
    T = torch.full((X.shape[0], r), float("nan"), device="cuda")
    none = torch.empty((G, 0, r) if trans[2] else (G, r, 0), dtype=dtype, device="cuda")
    am.amulet_adapters_mm(X, None, A, none, i32(at), T, torch.empty(X.shape[0], 0, dtype=dtype, device="cuda"), scales=scales.cuda(), trans_a=trans[1], trans_b=trans[2])
    assert am.amulet_recent_kernel().split()[0] == "adapters_down"
    a = A.double().transpose(1, 2) if trans[1] else A.double()
    want = torch.zeros(X.shape[0], r, dtype=torch.float64, device="cuda")
    for g, (i, j) in enumerate(zip(at, at[1:])):
        want[i:j] = float(scales[g]) * (X[i:j].double() @ a[g])
    assert torch.equal(T.double(), want)


# 225 segments: rows without an adapter, 90 segments of none, 120 of one to three rows with and without adapters, 10 of none, four long ones
CROWD = [70] + [0] * 90 + [1 + i % 3 for i in range(120)] + [0] * 10 + [900, 1100, 700, 1000]
CROWD_OF = [-1] + [i % 6 for i in range(90)] + [i * 5 % 7 - 1 for i in range(120)] + [0] * 10 + [5, 2, 0, 3]


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (FP16, F32)])
@pytest.mark.parametrize("trans", [ALONG, ACROSS])
@pytest.mark.parametrize("tile,N,K,r", [("64x64", 264, 136, 16), ("64x64", 520, 136, 100), ("128x128", 4104, 136, 16), ("128x128", 4104, 136, 128), ("256x256", 4104, 1032, 16), ("256x256", 4104, 1032, 72),
                                        ("256x256", 4104, 1032, 128)])
def test_more_segments_than_a_list_holds(am, tile, N, K, r, trans, dtype, out):
    """A tile that meets more than 64 segments, whose first 64 have no rows to add, with one and several passes over the ranks."""
    print("crowd", tile, N, K, r, trans, dtype, flush=True)
    assert sum(CROWD) >= 16 * len(CROWD) and len(CROWD) == len(CROWD_OF)
    name, R, want = run_mm(am, K + r, CROWD, CROWD_OF, 6, N, K, r, dtype, out, trans, spare=9)
    assert name == "adapters_" + tile
    off = (R - want).abs()
    assert float(off.max()) <= LIMIT, int((off > LIMIT).sum())


# ---- the matrices' gradients: sums of a wave are below 2^13 (step 2^-11), of a row's product by all but the first of T's pieces some steps: at most
# 157 instructions' worth of rows (20000 in four waves) by two stand-ins, 0.15; the waves' and the pieces' sums are joined exactly

OUTER = [([1], None, 1, 1, 1), ([31, 32, 33], None, 3, 24, 8), ([127, 128, 129], None, 3, 130, 17), ([511, 512, 513, 1024], None, 4, 64, 16), ([4000], None, 1, 256, 16),
         ([20000, 100], None, 2, 64, 8), ([700, 31, 1, 300, 0, 1500], [1, 0, 1, 1, 0, 0], 2, 264, 64), ([9] * 148, [i % 3 for i in range(148)], 3, 320, 40), ([5000, 5001, 4999, 1384], None, 4, 1024, 33),
         ([2047, 2049, 1, 8191], [0, 1, 0, 1], 2, 4096, 16), ([16384], None, 1, 512, 128)]


@pytest.mark.parametrize("lent", [0, 1 << 26])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("trans_r", [False, True])
@pytest.mark.parametrize("sizes,which,G,N,r", OUTER)
def test_every_row_counts(am, sizes, which, G, N, r, trans_r, dtype, lent):
    print("rows", sizes[:6], G, N, r, trans_r, dtype, lent, flush=True)
    ws = torch.full((lent,), 255, dtype=torch.uint8, device="cuda") if lent else None
    shape = (G, r, N) if trans_r else (G, N, r)
    for problem in (outer_problem, fine_problem):
        X, T, at, who = problem(N + r, sizes, which, G, N, r)
        X, T = X.cuda().to(dtype), T.cuda()
        R, R16 = torch.full(shape, float("nan"), device="cuda"), torch.full(shape, float("nan"), dtype=dtype, device="cuda")
        am.amulet_adapters_wgrad(X, T, i32(at), R, ws, adapters=None if which is None else i32(which), trans_r=trans_r)
        am.amulet_adapters_wgrad(X, T, i32(at), R16, ws, adapters=None if which is None else i32(which), trans_r=trans_r)
        want = outer_answer(X, T, at, who, G)
        off = ((R.transpose(1, 2) if trans_r else R).double() - want).abs()
        limit = fine_limit(at, who, G, T) if problem is fine_problem else 0.25
        assert float(off.max()) <= limit, (problem.__name__, int((off > limit).sum()))
        assert torch.equal(R16, R.to(dtype)), problem.__name__
