"""A mixture-of-experts layer's operators against their definitions in 64 bits: the router, the products by groups of rows
and their gradients, the sum back to the tokens, the fp8 quantiser and products.

Bounds are of the arithmetic, not of what was seen.  A product of two 16-bit values is exact in fp32; a sum of n of them in
fp32, in any order, is within n 2^-24 of the sum of their magnitudes (twice that is allowed for the additions inside a
matrix instruction), and the result is rounded once: half a unit in its last place.  fp8: the instruction's sum of 128
products may drop what is below 2^-16 of the largest of each."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, FP16: 2.0 ** -11}
LEAST = {F32: 2.0 ** -126, BF16: 2.0 ** -126, FP16: 2.0 ** -25}     # half the step of the smallest values


@pytest.fixture(scope="module")
def am():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2305_08872_amd as am
    am.load_library()
    return am


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, pad=0, shift=0, scale=1.0):
    """Normal values; pad: elements between rows; shift: elements that the first value lies off its allocation."""
    *lead, rows, cols = shape
    n = math.prod(lead) * rows * (cols + pad)
    x = torch.empty(shift + n, device="cuda").normal_(0, scale, generator=g).to(dtype)
    x[:shift] = math.nan                       # what lies around the operand is not to be used
    v = x[shift:].view(*lead, rows, cols + pad)
    v[..., cols:] = math.nan
    return v[..., :cols]


def within(got, want, slack, what):
    """|got - want| <= slack + the rounding of the result, everywhere; nan where it is wanted."""
    got64 = got.double()
    assert torch.equal(torch.isnan(got64), torch.isnan(want)), what
    limit = slack + HALF_ULP[got.dtype] * (want.abs() + slack) + LEAST[got.dtype]
    off = (got64 - want).abs()
    bad = (off > limit) & ~torch.isnan(want) & (got64 != want)
    assert not bad.any(), "%s: %d off, worst %.3g over its limit" % (what, int(bad.sum()), float((off / limit)[~torch.isnan(want)].max()))


def offsets_of(sizes, first=0):
    at = [first]
    for n in sizes:
        at.append(at[-1] + n)
    return at


def ref_rows(A, B, at, M, rows, trans_b):
    """(sums, sums of magnitudes) in 64 bits; zeros for rows of no group."""
    R = torch.zeros(M, B.shape[1] if trans_b else B.shape[2], dtype=torch.float64, device="cuda")
    S = torch.zeros_like(R)
    for g, (i, j) in enumerate(zip(at, at[1:])):
        if j <= i:
            continue
        b = B[g].double().t().contiguous() if trans_b else B[g].double()
        a = A[i:j].double()
        if rows is not None:
            r = rows[i:j].long()
            ok = (r >= 0) & (r < A.shape[0])
            a = A.double()[r.clamp(0, A.shape[0] - 1)]
            a[~ok] = 0
        R[i:j] = a @ b
        S[i:j] = a.abs() @ b.abs()
    return R, S


# sizes of groups, N, K: empty groups, single rows, one k, ends inside units, stages and tiles
SHAPES = [
    ([1], 1, 1), ([0, 1, 0], 8, 8), ([3, 0, 2], 17, 33), ([5, 9, 1, 0, 2], 64, 64), ([16, 16], 32, 128), ([7], 130, 200),
    ([20, 31, 0, 25], 96, 127), ([30, 30], 129, 65), ([61, 40, 70], 200, 192), ([64], 100, 71), ([50, 64], 128, 640),
    ([100, 130, 90], 260, 136), ([300, 1, 200], 129, 321), ([128, 256], 256, 64), ([700], 72, 1000),
    ([2100, 1996], 4000, 72), ([2300, 0, 1800], 4099, 130), ([4096], 4096, 193), ([1500, 1700], 1000, 520), ([256], 4096, 4096),
    ([4096], 8192, 1030), ([2500, 0, 1700], 8200, 1000), ([4100], 8195, 1024),
]


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (FP16, FP16)])
@pytest.mark.parametrize("sizes,N,K", SHAPES)
def test_products_by_rows(am, sizes, N, K, dtype, out, trans_b):
    print("grouped_mm", sizes, N, K, dtype, out, trans_b, flush=True)
    g = gen(N * 1000 + K)
    M = sum(sizes)
    A = normal(g, M, K, dtype=dtype)
    B = normal(g, len(sizes), *((N, K) if trans_b else (K, N)), dtype=dtype)
    at = offsets_of(sizes)
    R = torch.full((M, N), math.nan, dtype=out, device="cuda")
    am.amulet_grouped_mm(A, B, torch.tensor(at, dtype=torch.int32, device="cuda"), R, trans_b=trans_b)
    want, S = ref_rows(A, B, at, M, None, trans_b)
    within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")


def test_the_shapes_above_run_every_kernel(am):
    seen = set()
    for sizes, N, K in SHAPES:
        M = sum(sizes)
        A, B = torch.zeros(M, K, dtype=BF16, device="cuda"), torch.zeros(len(sizes), K, N, dtype=BF16, device="cuda")
        R = torch.ones(M, N, dtype=BF16, device="cuda")
        am.amulet_grouped_mm(A, B, torch.tensor(offsets_of(sizes), dtype=torch.int32, device="cuda"), R)
        seen.add(am.amulet_recent_kernel().split()[0])
        assert not R.any()
    assert seen == {"grouped_mm_" + t for t in ("256x256", "128x128", "64x128", "64x64", "64x64_k2", "16x32")}


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("sizes,N,K", [([3, 2], 37, 75), ([40, 0, 30], 136, 130), ([150, 150], 265, 200), ([4100], 4104, 200), ([4100], 8199, 1003)])
def test_products_by_rows_of_views(am, sizes, N, K, pad, shift, trans_b):
    """Rows apart, at odd addresses, the groups' matrices apart, R a view too; nothing beside the operands is used or written."""
    print("views", sizes, N, K, pad, shift, trans_b, flush=True)
    g = gen(pad * 10 + shift + K)
    M, G = sum(sizes), len(sizes)
    A = normal(g, M, K, dtype=BF16, pad=pad, shift=shift)
    B = normal(g, G, *((N, K) if trans_b else (K, N)), dtype=BF16, pad=pad, shift=shift)
    R = torch.full((shift + M * (N + pad),), 7.0, dtype=BF16, device="cuda")
    view = R[shift:].view(M, N + pad)[:, :N]
    at = offsets_of(sizes)
    am.amulet_grouped_mm(A, B, torch.tensor(at, dtype=torch.int32, device="cuda"), view, trans_b=trans_b)
    want, S = ref_rows(A, B, at, M, None, trans_b)
    within(view, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")
    assert (R[:shift] == 7).all() and (R[shift:].view(M, N + pad)[:, N:] == 7).all()


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("first,sizes,rest,N,K,tokens", [(0, [3, 0, 5], 0, 40, 64, 4), (2, [20, 40], 9, 70, 96, 31), (0, [0, 0], 12, 16, 8, 3), (5, [200, 330, 120], 40, 200, 260, 100),
                                                         (300, [2000, 2100], 290, 4000, 136, 777), (300, [2000, 2100], 290, 8200, 1000, 777)])
def test_gathered_rows_and_rows_of_no_group(am, first, sizes, rest, N, K, tokens, trans_b):
    """Row indexes that name no row stand for zeros; rows before the first group and behind the last are zeros."""
    print("gather", first, sizes, rest, N, K, tokens, trans_b, flush=True)
    g = gen(N + K)
    M = first + sum(sizes) + rest
    A = normal(g, tokens, K, dtype=BF16)
    B = normal(g, len(sizes), *((N, K) if trans_b else (K, N)), dtype=BF16)
    rows = torch.randint(0, tokens, (M,), generator=g, device="cuda", dtype=torch.int32)
    rows[:: 7] = -1
    rows[3:: 11] = tokens
    at = offsets_of(sizes, first)
    R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
    am.amulet_grouped_mm(A, B, torch.tensor(at, dtype=torch.int32, device="cuda"), R, rows=rows, trans_b=trans_b)
    want, S = ref_rows(A, B, at, M, rows, trans_b)
    within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")


# the largest tiles fill the chip once and a bit: their last columns go to smaller tiles in a second launch
@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("first,sizes,rest,N,K,tokens", [(0, [1300, 1250, 1200, 1250], 0, 4099, 1203, 0), (300, [1024, 1024, 1280, 1024], 10, 4096, 1280, 900), (0, [4096], 0, 4608, 1088, 0)])
def test_one_round_of_tiles_and_a_bit(am, first, sizes, rest, N, K, tokens, trans_b):
    print("a round and a bit", first, sizes, rest, N, K, tokens, trans_b, flush=True)
    g = gen(N + K)
    M = first + sum(sizes) + rest
    A = normal(g, tokens or M, K, dtype=BF16)
    B = normal(g, len(sizes), *((N, K) if trans_b else (K, N)), dtype=BF16)
    rows = torch.randint(0, tokens, (M,), generator=g, device="cuda", dtype=torch.int32) if tokens else None
    at = offsets_of(sizes, first)
    off = torch.tensor(at, dtype=torch.int32, device="cuda")
    R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
    am.amulet_grouped_mm(A, B, off, R, rows=rows, trans_b=trans_b)
    assert am.amulet_recent_kernel().split()[0] == "grouped_mm_256x256"
    want, S = ref_rows(A, B, at, M, rows, trans_b)
    within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")
    again = torch.full_like(R, math.nan)
    am.amulet_grouped_mm(A, B, off, again, rows=rows, trans_b=trans_b)
    assert torch.equal(again, R)


@pytest.mark.parametrize("trans_b", [False, True])
def test_fp8_one_round_of_tiles_and_a_bit(am, trans_b):
    g = gen(77)
    M, N, K = 4096, 4608, 2100
    A, sa, B, sb = fp8_operands(g, M, K, (1, N, K) if trans_b else (1, K, N))
    R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
    am.amulet_mm_fp8(A, sa, B[0], sb[0], R, trans_b=trans_b)
    assert am.amulet_recent_kernel().split()[0] == "mm_fp8_256x256"
    check_fp8(R, A, sa, B, sb, [0, M], None, trans_b)


def test_many_groups_and_offsets_out_of_range(am):
    """More groups than a wave has lanes; offsets past either end count as the end."""
    g = gen(3)
    sizes = [(i * 7) % 5 for i in range(333)]
    M, N, K = sum(sizes), 48, 72
    A, B = normal(g, M, K, dtype=FP16), normal(g, len(sizes), K, N, dtype=FP16)
    at = offsets_of(sizes)
    R = torch.empty(M, N, dtype=F32, device="cuda")
    am.amulet_grouped_mm(A, B, torch.tensor(at, dtype=torch.int32, device="cuda"), R)
    want, S = ref_rows(A, B, at, M, None, False)
    within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")
    wide = torch.tensor([-5, 10, 10, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    am.amulet_grouped_mm(A, B[:3], wide, R)
    want, S = ref_rows(A, B[:3], [0, 10, 10, M], M, None, False)
    within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")


def test_nothing_to_sum_and_nothing_to_write(am):
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    R = torch.ones(4, 6, dtype=BF16, device="cuda")
    am.amulet_grouped_mm(torch.empty(4, 0, dtype=BF16, device="cuda"), torch.empty(1, 0, 6, dtype=BF16, device="cuda"), off, R)
    assert not R.any()
    R.fill_(1)
    am.amulet_grouped_mm(torch.empty(0, 8, dtype=BF16, device="cuda"), torch.ones(1, 8, 6, dtype=BF16, device="cuda"), off, R,
                         rows=torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert not R.any()
    R.fill_(1)
    am.amulet_grouped_mm(torch.ones(4, 8, dtype=BF16, device="cuda"), torch.empty(0, 8, 6, dtype=BF16, device="cuda"), off[:1], R)
    assert not R.any()
    W = torch.ones(1, 8, 6, dtype=BF16, device="cuda")
    am.amulet_grouped_mm_wgrad(torch.empty(0, 8, dtype=BF16, device="cuda"), torch.empty(0, 6, dtype=BF16, device="cuda"), off * 0, W)
    assert not W.any()
    am.amulet_grouped_mm(torch.empty(0, 8, dtype=BF16, device="cuda"), W, off * 0, torch.empty(0, 6, dtype=BF16, device="cuda"))


def test_infinities_and_nan_reach_their_own_outputs_only(am):
    """A NaN in a row, a column or a matrix, and in the k next to a ragged end: no other output has one."""
    g = gen(9)
    for K, N, sizes in [(70, 50, [5, 6]), (200, 300, [150, 140]), (65, 4000, [2100, 2100]), (1001, 8200, [2100, 2100])]:
        M = sum(sizes)
        A, B = normal(g, M, K, dtype=BF16), normal(g, 2, K, N, dtype=BF16)
        A[2, K - 1] = math.nan
        A[M - 1, 0] = math.inf
        B[0, K - 1, N - 1] = math.nan
        at = offsets_of(sizes)
        for trans_b in (False, True):
            R = torch.empty(M, N, dtype=F32, device="cuda")
            am.amulet_grouped_mm(A, B.transpose(1, 2).contiguous() if trans_b else B, torch.tensor(at, dtype=torch.int32, device="cuda"), R, trans_b=trans_b)
            bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
            bad[2], bad[M - 1], bad[:sizes[0], N - 1] = True, True, True
            assert torch.equal(~torch.isfinite(R), bad)


@pytest.mark.parametrize("sizes,N,K", [([1], 8, 65), ([7], 130, 200), ([64], 100, 71), ([50, 64], 128, 616), ([300, 1, 200], 129, 321), ([700], 72, 1000), ([2100, 1996], 4000, 72)])
def test_an_infinity_near_a_ragged_end_stays_one(am, sizes, N, K):
    """The k before a ragged end, each infinite in one operand and 2 in the other: every sum is infinite and none is NaN, whichever
    stages have that k."""
    M, G = sum(sizes), len(sizes)
    off = torch.tensor(offsets_of(sizes), dtype=torch.int32, device="cuda")
    for k in {K - 1, K - K % 64, K - K % 64 - 1, max(0, K - 64), max(0, K - 65)}:
        A, B = torch.full((M, K), 2.0, dtype=BF16, device="cuda"), torch.ones(G, K, N, dtype=BF16, device="cuda")
        A[::2, k] = math.inf
        want = torch.full((M, N), 2.0 * K, device="cuda")
        want[::2] = math.inf
        for trans_b in (False, True):
            b = B.transpose(1, 2).contiguous() if trans_b else B
            R = torch.empty(M, N, dtype=F32, device="cuda")
            am.amulet_grouped_mm(A, b, off, R, trans_b=trans_b)
            assert torch.equal(R, want)
        B[:, k, ::3] = -math.inf
        A[:, k] = 2.0
        want = torch.full((M, N), 2.0 * K, device="cuda")
        want[:, ::3] = -math.inf
        for trans_b in (False, True):
            b = B.transpose(1, 2).contiguous() if trans_b else B
            R = torch.empty(M, N, dtype=F32, device="cuda")
            am.amulet_grouped_mm(A, b, off, R, trans_b=trans_b)
            assert torch.equal(R, want)


@pytest.mark.parametrize("trans_r", [False, True])
@pytest.mark.parametrize("dtype,out,space", [(BF16, BF16, 0), (BF16, F32, 1 << 24), (FP16, FP16, 1 << 30)])
@pytest.mark.parametrize("sizes,N,K,tokens", [([1], 1, 1, 0), ([3, 0, 2], 17, 33, 0), ([64, 0, 128], 64, 72, 0), ([65, 200, 1], 129, 130, 50), ([700, 3, 0, 90], 136, 264, 333),
                                              ([9000], 64, 72, 0), ([5000, 2600], 100, 61, 1000), ([300, 130], 3000, 2900, 0), ([70, 0, 250], 2900, 2955, 99)])
def test_gradients_of_the_matrices(am, sizes, N, K, tokens, dtype, out, space, trans_r):
    print("wgrad", sizes, N, K, tokens, dtype, out, space, trans_r, flush=True)
    g = gen(N + 7 * K)
    M, G = sum(sizes) + 5, len(sizes)
    at = offsets_of(sizes, 2)
    A = normal(g, tokens or M, K, dtype=dtype, pad=N % 3)
    D = normal(g, M, N, dtype=dtype, shift=K % 2)
    rows = None
    if tokens:
        rows = torch.randint(0, tokens, (M,), generator=g, device="cuda", dtype=torch.int32)
        rows[::9] = -1
    R = torch.full((G, N, K) if trans_r else (G, K, N), math.nan, dtype=out, device="cuda")
    ws = torch.full((space // 4,), math.nan, device="cuda") if space else None
    am.amulet_grouped_mm_wgrad(A, D, torch.tensor(at, dtype=torch.int32, device="cuda"), R, ws, rows=rows, trans_r=trans_r)
    want = torch.zeros(R.shape, dtype=torch.float64, device="cuda")
    S = torch.zeros_like(want)
    for e, (i, j) in enumerate(zip(at, at[1:])):
        d = D[i:j].double()
        a = A[i:j].double()
        if rows is not None:
            r = rows[i:j].long()
            a = A.double()[r.clamp(min=0)]
            a[r < 0] = 0
        w = a.t().contiguous() @ d
        s = a.abs().t().contiguous() @ d.abs()
        want[e], S[e] = (w.t(), s.t()) if trans_r else (w, s)
    within(R, want, 2 * (max(sizes) + 8) * 2.0 ** -24 * S, "dB")
    again = torch.empty_like(R)
    am.amulet_grouped_mm_wgrad(A, D, torch.tensor(at, dtype=torch.int32, device="cuda"), again, ws, rows=rows, trans_r=trans_r)
    assert torch.equal(R, again)


def test_gradients_of_the_products_against_differences(am):
    """f = sum C * (A B by groups): its change along a direction in A and in B, in 64 bits, against the gradients."""
    g = gen(21)
    sizes, N, K = [40, 0, 25], 48, 56
    M, at = sum(sizes), offsets_of(sizes)
    off = torch.tensor(at, dtype=torch.int32, device="cuda")
    A, B, C = normal(g, M, K, dtype=BF16), normal(g, 3, K, N, dtype=BF16), normal(g, M, N, dtype=BF16)
    dA, dB = torch.empty(M, K, device="cuda"), torch.empty(3, K, N, device="cuda")
    am.amulet_grouped_mm(C, B, off, dA, trans_b=True)
    am.amulet_grouped_mm_wgrad(A, C, off, dB)
    VA, VB = normal(g, M, K).double(), normal(g, 3, K, N).double()

    def f(a, b):
        return sum(float((C[i:j].double() * (a[i:j] @ b[e])).sum()) for e, (i, j) in enumerate(zip(at, at[1:])))
    h = 2.0 ** -10
    a, b = A.double(), B.double()
    for got, num in [((dA.double() * VA).sum(), (f(a + h * VA, b) - f(a - h * VA, b)) / (2 * h)), ((dB.double() * VB).sum(), (f(a, b + h * VB) - f(a, b - h * VB)) / (2 * h))]:
        # (f is linear in each: differences have no error of their own but the 64-bit roundings'; fp32 sums of 65 terms)
        assert abs(float(got) - num) <= 1e-5 * (dA.double().abs().sum() + dB.double().abs().sum()) * 1e-1


# ------------------------------------------------------------------------------------------------ router

def ref_route(logits, k, norm):
    """experts, weights, place, tokens, offsets on the host, token by token."""
    T, E = logits.shape
    x = logits.double().cpu()
    experts, weights = torch.full((T, k), -1, dtype=torch.int32), torch.zeros(T, k, dtype=torch.float64)
    pairs = [[] for _ in range(E)]
    for t, row in enumerate(x.tolist()):
        order = sorted((e for e in range(E) if row[e] > -math.inf), key=lambda e: (-row[e], e))[:k]
        if not order:
            continue
        most = row[order[0]]
        term = (lambda v: 1.0 if v == math.inf else 0.0) if most == math.inf else (lambda v: math.exp(v - most))
        total = sum(term(row[e]) for e in (order if norm else [e for e in range(E) if row[e] > -math.inf]))
        for j, e in enumerate(order):
            experts[t, j], weights[t, j] = e, term(row[e]) / total
            pairs[e].append(t * k + j)
    place, tokens, offsets = torch.full((T * k,), -1, dtype=torch.int32), torch.full((T * k,), -1, dtype=torch.int32), [0]
    for e in range(E):
        for n, p in enumerate(pairs[e]):
            place[p], tokens[offsets[-1] + n] = offsets[-1] + n, p // k
        offsets.append(offsets[-1] + len(pairs[e]))
    return experts, weights, place.view(T, k), tokens, torch.tensor(offsets, dtype=torch.int32)


def run_route(am, logits, k, norm):
    T, E = logits.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    experts, place = torch.full((T, k), 99, **i32), torch.full((T, k), 99, **i32)
    tokens, offsets = torch.full((T * k,), 99, **i32), torch.full((E + 1,), 99, **i32)
    weights = torch.full((T, k), math.nan, device="cuda")
    ws = torch.full((am.amulet_route_workspace_bytes(T, E),), 99, dtype=torch.uint8, device="cuda")
    am.amulet_route(logits, experts, weights, place, tokens, offsets, ws, norm=norm)
    return experts, weights, place, tokens, offsets


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16, FP16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (8, 64, 6), (64, 60, 8), (65, 60, 4), (130, 128, 8), (1000, 16, 16), (777, 256, 8), (100, 300, 5), (300, 1024, 64), (40, 20, 20), (20000, 9, 3)])
def test_route(am, T, E, k, dtype, norm):
    print("route", T, E, k, dtype, norm, flush=True)
    g = gen(T + E)
    x = normal(g, T, E, pad=T % 3).to(dtype)
    if T > 1:
        # masked experts, masked tokens, ties, zeros of both signs, the type's lowest value, NaN and infinities
        x[torch.empty(T, E, device="cuda").uniform_(generator=g) < 0.2] = -math.inf
        x[1::5] = -math.inf
        x[2::7] = 0.0
        x[2::7, ::2] = -0.0
        x[3::11] = torch.finfo(dtype).min
        x[4::13, 0] = math.nan
        x[5::17, E // 2] = math.inf
    got = run_route(am, x, k, norm)
    want = ref_route(x, k, norm)
    for name, a, b in zip(("experts", "weights", "place", "tokens", "offsets"), got, want):
        if name == "weights":
            # one exp (2 units in the last place), a sum of E of them and a division
            assert ((a.cpu().double() - b).abs() <= (E + 8) * 2.0 ** -23 * b + 2.0 ** -126).all()
        else:
            assert torch.equal(a.cpu(), b), name


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16, FP16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (8, 64, 6), (130, 128, 8), (50, 300, 30), (33, 1024, 64)])
def test_route_grad(am, T, E, k, dtype, norm):
    print("route_grad", T, E, k, dtype, norm, flush=True)
    g = gen(T * E)
    x = normal(g, T, E).to(dtype)
    if T > 1:
        x[torch.empty(T, E, device="cuda").uniform_(generator=g) < 0.2] = -math.inf
        x[1::5] = -math.inf
    experts, weights = run_route(am, x, k, norm)[:2]
    up = normal(g, T, k)
    dx = torch.full((T, E + 3), math.nan, dtype=dtype, device="cuda")[:, :E]
    am.amulet_route_grad(None if norm else x, experts, weights, up, dx, norm=norm)
    # the formula: dx = p (up - sum p up) with up at the chosen experts
    chosen = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    at, there = experts.clamp(min=0).long(), (experts >= 0).double()
    chosen.scatter_add_(1, at, there)
    spread = torch.zeros_like(chosen).scatter_add_(1, at, up.double() * there)
    x64 = x.double()
    keep = chosen > 0 if norm else x64 > -math.inf
    term = torch.where(keep, torch.exp(x64 - x64.masked_fill(~keep, -1e300).amax(1, keepdim=True)), 0.0)
    p = term / term.sum(1, keepdim=True).clamp(min=1e-300)
    want = p * (spread - (p * spread).sum(1, keepdim=True))
    slack = p * (E + 2 * k + 32) * 2.0 ** -23 * (spread.abs() + (p * spread.abs()).sum(1, keepdim=True))
    within(dx, want, slack, "dlogits")


@pytest.mark.parametrize("norm", [True, False])
def test_route_grad_against_differences(am, norm):
    g = gen(5)
    T, E, k = 12, 20, 4
    x = normal(g, T, E)
    experts, weights = run_route(am, x, k, norm)[:2]
    up = normal(g, T, k)
    dx = torch.empty(T, E, device="cuda")
    am.amulet_route_grad(x, experts, weights, up, dx, norm=norm)
    v = normal(g, T, E).double()

    def f(y):
        # (the choice held: a small step does not change it)
        w = torch.exp(y - y.amax(1, keepdim=True))
        c = w.gather(1, experts.long())
        return float((up.double() * c / (c if norm else w).sum(1, keepdim=True)).sum())
    h = 1e-5
    num = (f(x.double() + h * v) - f(x.double() - h * v)) / (2 * h)
    assert abs(float((dx.double() * v).sum()) - num) <= 1e-5 * float((dx.double() * v).abs().sum()) + 1e-8


# ------------------------------------------------------------------------------------------------ combine

@pytest.mark.parametrize("dtype", [F32, BF16, FP16])
@pytest.mark.parametrize("T,k,H,pad", [(1, 1, 1, 0), (5, 3, 7, 0), (8, 6, 512, 0), (33, 2, 130, 3), (64, 8, 1000, 0), (100, 5, 2048, 8), (7, 70, 96, 0)])
def test_combine_and_its_gradients(am, T, k, H, pad, dtype):
    print("combine", T, k, H, pad, dtype, flush=True)
    g = gen(T + H)
    rows = T * k + 3
    place = torch.randperm(rows, generator=g, device="cuda")[:T * k].view(T, k).int()
    place[torch.empty(T, k, device="cuda").uniform_(generator=g) < 0.2] = -1
    if T > 1:
        place[1] = -1
        place[0, 0] = rows                       # (names no row)
    Y, dR = normal(g, rows, H, dtype=dtype, pad=pad), normal(g, T, H, dtype=dtype, pad=pad)
    used = place[(place >= 0) & (place < rows)].long()
    spare = torch.ones(rows, dtype=torch.bool, device="cuda")
    spare[used] = False
    Y[spare] = math.nan                          # rows that no pair names are not read
    w = normal(g, T, k).contiguous()
    there = (place >= 0) & (place < rows)
    y = torch.where(there[:, :, None], Y.double()[place.clamp(0, rows - 1).long()], 0.0)
    for weights in (w, None):
        f = (w if weights is not None else torch.ones_like(w)).double() * there
        R = torch.full((T, H), math.nan, dtype=dtype, device="cuda")
        am.amulet_combine(Y, weights, place, R)
        within(R, (f[:, :, None] * y).sum(1), (k + 2) * 2.0 ** -24 * (f[:, :, None] * y).abs().sum(1), "R")
        dY = torch.full((rows, H + pad), 7.0, dtype=dtype, device="cuda")[:, :H]
        dw = torch.full((T, k), math.nan, device="cuda")
        am.amulet_combine_grad(Y, weights, place, dR, dY, dw)
        want = torch.full((rows, H), 7.0, dtype=torch.float64, device="cuda")
        want[place[there].long()] = (f[:, :, None] * dR.double()[:, None, :])[there]
        within(dY, want, torch.zeros_like(want), "dY")
        prod = y * dR.double()[:, None, :]
        within(dw, prod.sum(2), (H + 8) * 2.0 ** -24 * prod.abs().sum(2), "dweights")
        only = torch.full_like(dY, 7.0)
        am.amulet_combine_grad(None, weights, place, dR, only)
        assert torch.equal(only, dY)


# ------------------------------------------------------------------------------------------------ fp8

def ref_quantize(x, rows):
    """x G x M x K (64 bits of the 32-bit arithmetic: scale and its reciprocal are rounded as stated): (q, scales)."""
    G, M, K = x.shape
    p = torch.nn.functional.pad(x.float(), (0, -K % 128, 0, -M % rows))
    b = p.view(G, p.shape[1] // rows, rows, p.shape[2] // 128, 128)
    scale = torch.maximum(b.abs().amax((2, 4)).double().div(448.0).float(), torch.tensor(2.0 ** -126, device="cuda"))
    r = (1.0 / scale.double()).float()
    v = (b * r[:, :, None, :, None]).double()
    # to the nearest multiple of the step of its octave, ties to even
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    q = (torch.round(v / step) * step).reshape(p.shape)[:, :M, :K]
    return q, scale


@pytest.mark.parametrize("dtype", [F32, BF16, FP16])
@pytest.mark.parametrize("M,K,pad", [(1, 1, 0), (3, 128, 0), (17, 200, 0), (16, 1024, 8), (100, 257, 1), (33, 4096, 0), (5, 640, 0)])
def test_quantize_rows(am, M, K, pad, dtype):
    print("quantize", M, K, pad, dtype, flush=True)
    g = gen(M + K)
    x = normal(g, M, K, dtype=dtype, pad=pad)
    x[0, :128] = 0.0
    if M > 2:
        x[1] *= 1e-4
        x[2, K // 2] = 30000.0
    q = torch.empty(M, K + pad, dtype=torch.float8_e4m3fn, device="cuda")[:, :K]
    s = torch.full(((K + 127) // 128, M), math.nan, device="cuda")
    am.amulet_quantize_fp8(x, q, s)
    want, scale = ref_quantize(x[None], 1)
    assert torch.equal(s, scale[0].t())
    assert torch.equal(q.double(), want[0])


@pytest.mark.parametrize("dtype", [F32, BF16, FP16])
@pytest.mark.parametrize("G,M,K,pad", [(1, 1, 1, 0), (2, 128, 128, 0), (3, 200, 300, 0), (2, 100, 1000, 1), (1, 257, 640, 8)])
def test_quantize_blocks(am, G, M, K, pad, dtype):
    print("quantize blocks", G, M, K, pad, dtype, flush=True)
    x = normal(gen(M + K), G, M, K, dtype=dtype, pad=pad)
    x[0, :128, :128] = 0.0
    q = torch.empty(G, M, K + pad, dtype=torch.float8_e4m3fn, device="cuda")[:, :, :K]
    s = torch.full((G, (M + 127) // 128, (K + 127) // 128), math.nan, device="cuda")
    am.amulet_quantize_fp8_blocks(x, q, s)
    want, scale = ref_quantize(x, 128)
    assert torch.equal(s, scale)
    assert torch.equal(q.double(), want)


def test_quantize_keeps_what_is_not_finite_visible(am):
    x = torch.ones(2, 256, device="cuda")
    x[0, 3], x[1, 200] = math.nan, math.inf
    q, s = torch.empty(2, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(2, 2, device="cuda")
    am.amulet_quantize_fp8(x, q, s)
    f = q.float()
    assert torch.isnan(f[0, 3]) and int(torch.isnan(f).sum()) == 2 and torch.isnan(f[1, 200])
    assert s[1, 1] == math.inf and s[0, 0] == torch.tensor(1.0).div(448.0)


def fp8_operands(g, M, K, shape, pad=0):
    a = normal(g, M, K) * torch.where(torch.empty(K, device="cuda").uniform_(generator=g) < 0.05, 8.0, 1.0)
    b = normal(g, *shape)
    qa, sa = ref_quantize(a[None], 1)
    qb, sb = ref_quantize(b, 128)

    def store(q):
        x = torch.full(q.shape[:-1] + (q.shape[-1] + pad,), math.nan, device="cuda").to(torch.float8_e4m3fn)
        x[..., :q.shape[-1]] = q.float().to(torch.float8_e4m3fn)
        return x[..., :q.shape[-1]]
    return store(qa[0]), sa[0].t().contiguous(), store(qb), sb


def spread_scale(s, n, m):
    return s.double().repeat_interleave(128, -2)[..., :n, :].repeat_interleave(128, -1)[..., :m]


def check_fp8(R, A, sa, B, sb, at, rows, trans_b):
    M, K = R.shape[0], A.shape[1]
    av = A.double() * sa.t().double().repeat_interleave(128, 1)[:, :K]
    bv = B.double() * spread_scale(sb, B.shape[1], B.shape[2])
    want, S = ref_rows(av, bv, at, M, rows, trans_b)
    # largest products of each 128 k, of the values with their scales: 128 times 2^-16 of them may be dropped
    KB = sa.shape[0]
    pad = torch.nn.functional.pad
    amax = pad(av.abs(), (0, KB * 128 - K)).view(-1, KB, 128).amax(2)
    bk = bv.abs() if not trans_b else bv.abs().transpose(1, 2)
    bmax = pad(bk, (0, 0, 0, KB * 128 - K)).reshape(B.shape[0], KB, 128, -1).amax(2)
    D = ref_rows(amax, bmax.contiguous(), at, M, rows, False)[0]
    within(R, want, 128 * 2.0 ** -16 * D + 2 * (KB + 8) * 2.0 ** -24 * S, "R")


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("out", [F32, BF16, FP16])
@pytest.mark.parametrize("sizes,N,K,tokens", [([1], 1, 1, 0), ([3, 0, 2], 17, 33, 0), ([5, 9, 1], 64, 128, 7), ([16], 8200, 256, 0), ([20, 31, 0], 96, 127, 0), ([61, 40], 200, 500, 33),
                                              ([100, 130, 90], 260, 136, 0), ([300, 1, 200], 129, 1321, 400), ([2100, 1996], 4000, 200, 0), ([4096], 4100, 384, 1000), ([2100, 1996], 8200, 1001, 0), ([4096], 8195, 1408, 1000), ([256], 4096, 4096, 0)])
def test_fp8_products(am, sizes, N, K, tokens, out, trans_b):
    print("fp8", sizes, N, K, tokens, out, trans_b, flush=True)
    g = gen(N + K)
    M, G = sum(sizes), len(sizes)
    A, sa, B, sb = fp8_operands(g, tokens or M, K, (G, N, K) if trans_b else (G, K, N), pad=N % 3)
    rows = None
    if tokens:
        rows = torch.randint(0, tokens, (M,), generator=g, device="cuda", dtype=torch.int32)
        rows[::9] = -1
    at = offsets_of(sizes)
    R = torch.full((M, N), math.nan, dtype=out, device="cuda")
    am.amulet_grouped_mm_fp8(A, sa, B, sb, torch.tensor(at, dtype=torch.int32, device="cuda"), R, rows=rows, trans_b=trans_b)
    check_fp8(R, A, sa, B, sb, at, rows, trans_b)
    if G == 1 and not tokens:
        dense = torch.full_like(R, math.nan)
        am.amulet_mm_fp8(A, sa, B[0], sb[0], dense, trans_b=trans_b)
        assert torch.equal(dense, R)


# ------------------------------------------------------------------------------------------------ use

def test_on_another_stream_and_in_a_graph(am):
    """A layer's forward calls on a side stream and replayed from a graph, eager work between the replays."""
    g = gen(77)
    T, E, k, H, F = 100, 8, 2, 64, 96
    x, W = normal(g, T, H, dtype=BF16), normal(g, E, H, F, dtype=BF16, scale=H ** -0.5)
    logits = normal(g, T, E).contiguous()
    i32 = dict(dtype=torch.int32, device="cuda")
    experts, place, tokens, offsets = torch.empty(T, k, **i32), torch.empty(T, k, **i32), torch.empty(T * k, **i32), torch.empty(E + 1, **i32)
    weights, ws = torch.empty(T, k, device="cuda"), torch.empty(am.amulet_route_workspace_bytes(T, E), dtype=torch.uint8, device="cuda")
    Y, R = torch.empty(T * k, F, dtype=BF16, device="cuda"), torch.empty(T, F, dtype=BF16, device="cuda")

    def layer():
        am.amulet_route(logits, experts, weights, place, tokens, offsets, ws)
        am.amulet_grouped_mm(x, W, offsets, Y, rows=tokens)
        am.amulet_combine(Y, weights, place, R)
    layer()
    torch.cuda.synchronize()
    eager = R.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    R.fill_(0)
    with torch.cuda.stream(side):
        layer()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for n in range(4):
        logits.copy_(normal(g, T, E))
        x.copy_(normal(g, T, H, dtype=BF16))
        R.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = R.clone()
        layer()
        torch.cuda.synchronize()
        assert torch.equal(replayed, R)
        assert not torch.equal(R, eager)


def test_offsets_past_32_bits(am):
    """Rows whose byte offsets pass 4 GiB, gathered and in place."""
    K, N, rows = 4096, 64, 530000
    A = torch.zeros(rows, K, dtype=BF16, device="cuda")
    A[-1], A[-2], A[0] = 1.0, 2.0, 3.0
    B = torch.ones(1, K, N, dtype=BF16, device="cuda")
    at = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    R = torch.empty(3, N, device="cuda")
    am.amulet_grouped_mm(A, B, at, R, rows=torch.tensor([rows - 1, rows - 2, 0], dtype=torch.int32, device="cuda"))
    assert (R[0] == K).all() and (R[1] == 2 * K).all() and (R[2] == 3 * K).all()
    R = torch.empty(rows, N, dtype=BF16, device="cuda")
    am.amulet_grouped_mm(A, B, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), R)
    assert (R[-1] == K).all() and (R[-2] == 2 * K).all() and not R[1:-2].any()
    dB = torch.empty(1, K, N, device="cuda")
    D = torch.zeros(rows, N, dtype=BF16, device="cuda")
    D[-1], D[0] = 5.0, 1.0
    am.amulet_grouped_mm_wgrad(A, D, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), dB)
    assert (dB == 8).all()
