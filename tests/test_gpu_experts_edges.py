"""A mixture-of-experts layer's operators at the edges of their ranges, against 64 bits: operands of a few columns, no tokens, results
in views, offsets that do not ascend.  Bounds as in test_gpu_experts."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_experts import BF16, F32, FP16, check_fp8, fp8_operands, gen, normal, offsets_of, ref_rows, within  # noqa: E402


@pytest.fixture(scope="module")
def am():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2305_08872_amd as am
    am.load_library()
    return am


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# rows of a matrix shorter than the 16 bytes of a request, and a few k behind the last whole stage
@pytest.mark.parametrize("K", [64, 65, 66, 129, 131, 263])
@pytest.mark.parametrize("N", [1, 2, 3, 5, 7])
def test_matrices_of_a_few_columns(am, N, K):
    print("few columns", N, K, flush=True)
    g = gen(N * 1000 + K)
    for sizes in ([5], [3, 0, 70]):
        M, at = sum(sizes), offsets_of(sizes)
        off = i32(at)
        A, B = normal(g, M, K, dtype=BF16), normal(g, len(sizes), K, N, dtype=BF16)
        R = torch.full((M, N), math.nan, device="cuda")
        am.amulet_grouped_mm(A, B, off, R)
        want, S = ref_rows(A, B, at, M, None, False)
        within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")
        A8, sa, B8, sb = fp8_operands(g, M, K, (len(sizes), K, N))
        R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
        am.amulet_grouped_mm_fp8(A8, sa, B8, sb, off, R)
        check_fp8(R, A8, sa, B8, sb, at, None, False)


@pytest.mark.parametrize("M", [65, 66, 129, 700])
@pytest.mark.parametrize("K,N", [(1, 1), (2, 40), (3, 3), (300, 1), (7, 2)])
def test_gradients_of_matrices_of_a_few_columns(am, M, K, N):
    print("gradients, few columns", M, K, N, flush=True)
    g = gen(M + K + N)
    A, D = normal(g, M, K, dtype=FP16), normal(g, M, N, dtype=FP16)
    for sizes in ([M], [M - 64, 64], [M - 1, 0, 1]):
        at = offsets_of(sizes)
        ws = torch.full((1 << 20,), math.nan, device="cuda")
        for trans_r in (False, True):
            R = torch.full((len(sizes), N, K) if trans_r else (len(sizes), K, N), math.nan, device="cuda")
            am.amulet_grouped_mm_wgrad(A, D, i32(at), R, ws, trans_r=trans_r)
            for e, (i, j) in enumerate(zip(at, at[1:])):
                a, d = A[i:j].double(), D[i:j].double()
                w, s = a.t().contiguous() @ d, a.abs().t().contiguous() @ d.abs()
                within(R[e], w.t() if trans_r else w, 2 * (M + 8) * 2.0 ** -24 * (s.t() if trans_r else s), "dB")


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("E,k", [(1, 1), (8, 2), (200, 8), (1000, 64)])
def test_no_tokens(am, E, k, norm):
    """A batch without tokens: no expert has a row.  The offsets say so to the products, which write zeros."""
    print("no tokens", E, k, norm, flush=True)
    none = dict(dtype=torch.int32, device="cuda")
    for dtype in (F32, BF16, FP16):
        offsets = torch.full((E + 1,), 99, **none)
        logits = torch.empty(0, E, dtype=dtype, device="cuda")
        experts, weights = torch.empty(0, k, **none), torch.empty(0, k, device="cuda")
        place, tokens = torch.empty(0, k, **none), torch.empty(0, **none)
        am.amulet_route(logits, experts, weights, place, tokens, offsets, norm=norm)
        assert not offsets.any()
        am.amulet_route_grad(logits, experts, weights, torch.empty(0, k, device="cuda"), torch.empty_like(logits), norm=norm)
    x, W = torch.empty(0, 16, dtype=BF16, device="cuda"), torch.ones(E, 16, 24, dtype=BF16, device="cuda")
    y, R = torch.empty(0, 24, dtype=BF16, device="cuda"), torch.empty(0, 24, dtype=BF16, device="cuda")
    am.amulet_grouped_mm(x, W, offsets, y, rows=tokens)
    am.amulet_combine(y, weights, place, R)
    am.amulet_combine_grad(y, weights, place, R, y, weights)
    dW = torch.ones_like(W)
    am.amulet_grouped_mm_wgrad(x, y, offsets, dW, rows=tokens)
    assert not dW.any()
    am.amulet_quantize_fp8(x, torch.empty(0, 16, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(1, 0, device="cuda"))


def test_layer_without_tokens(am):
    """The example layer on an empty batch: outputs without rows, gradients that are zeros."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import experts_layer
    layer = experts_layer.Layer(32, 48, 4, 2)
    x = torch.empty(0, 32, dtype=BF16, device="cuda")
    out = layer.forward(x)
    dx, drouter, dw1, dw2 = layer.backward(out)
    assert out.shape == dx.shape == (0, 32)
    assert not drouter.any() and not dw1.any() and not dw2.any()
    layer.quantize()
    assert layer.forward_8bit(x).shape == (0, 32)


# The largest tiles fill the chip once and a bit, and the columns end inside a tile, a unit and a stage: the second launch's too.
@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("first,sizes,rest,N,K,tokens", [(0, [4096], 0, 4500, 1203, 0), (0, [4096], 0, 4367, 1211, 0), (5, [2000, 2100], 9, 4501, 1211, 777)])
def test_the_last_columns_of_ragged_products(am, first, sizes, rest, N, K, tokens, trans_b):
    print("last columns", first, sizes, rest, N, K, tokens, trans_b, flush=True)
    g = gen(N + K)
    M = first + sum(sizes) + rest
    A = normal(g, tokens or M, K, dtype=BF16)
    B = normal(g, len(sizes), *((N, K) if trans_b else (K, N)), dtype=BF16)
    rows = torch.randint(-1, tokens + 1, (M,), generator=g, device="cuda", dtype=torch.int32) if tokens else None
    at = offsets_of(sizes, first)
    R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
    am.amulet_grouped_mm(A, B, i32(at), R, rows=rows, trans_b=trans_b)
    assert am.amulet_recent_kernel() == "grouped_mm_256x256 rows %d last_columns 128" % M
    want, S = ref_rows(A, B, at, M, rows, trans_b)
    within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")
    again = torch.full_like(R, math.nan)
    am.amulet_grouped_mm(A, B, i32(at), again, rows=rows, trans_b=trans_b)
    assert torch.equal(again, R)


@pytest.mark.parametrize("trans_b", [False, True])
def test_the_last_columns_of_a_ragged_8_bit_product(am, trans_b):
    g = gen(78)
    M, N, K = 4096, 4501, 2111
    A, sa, B, sb = fp8_operands(g, M, K, (1, N, K) if trans_b else (1, K, N))
    R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
    am.amulet_mm_fp8(A, sa, B[0], sb[0], R, trans_b=trans_b)
    assert am.amulet_recent_kernel() == "mm_fp8_256x256 rows %d last_columns 128" % M
    check_fp8(R, A, sa, B, sb, [0, M], None, trans_b)


def matrices(layout, G, rows, cols, dtype):
    """(storage filled with sevens, G x rows x cols of it): with a pitch, without the last row's padding, the rows of all matrices in turn."""
    if layout == "turn":
        s = torch.full((rows, G, cols + 1), 7.0, device="cuda").to(dtype)
        return s, s.permute(1, 0, 2)[:, :, :cols]
    ld = cols + 3
    apart = rows * ld + 5 if layout == "pitch" else (rows - 1) * ld + cols
    s = torch.full((1 + (G - 1) * apart + rows * ld,), 7.0, device="cuda").to(dtype)
    return s, s.as_strided((G, rows, cols), (apart, ld, 1), 1)


@pytest.mark.parametrize("layout", ["pitch", "tight", "turn"])
@pytest.mark.parametrize("sizes,K,N,space", [([40, 0, 33], 37, 21, 0), ([6000, 2000], 70, 45, 1 << 24), ([300, 200], 300, 260, 0)])
@pytest.mark.parametrize("out", [BF16, F32])
def test_gradients_into_views(am, sizes, K, N, space, out, layout):
    """The results' rows and matrices apart: sums over ranges of the rows too.  Nothing beside them is written."""
    print("gradients into", layout, sizes, K, N, space, out, flush=True)
    g = gen(K + N)
    M, G, at = sum(sizes), len(sizes), offsets_of(sizes)
    A, D = normal(g, M, K, dtype=BF16), normal(g, M, N, dtype=BF16)
    ws = torch.full((space // 4,), math.nan, device="cuda") if space else None
    for trans_r in (False, True):
        store, R = matrices(layout, G, *((N, K) if trans_r else (K, N)), out)
        am.amulet_grouped_mm_wgrad(A, D, i32(at), R, ws, trans_r=trans_r)
        assert ("parts" in am.amulet_recent_kernel()) == (space > 0)
        for e, (i, j) in enumerate(zip(at, at[1:])):
            a, d = A[i:j].double(), D[i:j].double()
            w, s = a.t().contiguous() @ d, a.abs().t().contiguous() @ d.abs()
            within(R[e], w.t() if trans_r else w, 2 * (max(sizes) + 8) * 2.0 ** -24 * (s.t() if trans_r else s), "dB")
        R.fill_(7.0)
        assert (store == 7).all()


@pytest.mark.parametrize("layout", ["pitch", "tight", "turn"])
def test_quantised_matrices_into_views(am, layout):
    G, M, K = 3, 200, 300
    x = normal(gen(8), G, M, K, dtype=BF16)
    q, s = torch.empty(G, M, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(G, 2, 3, device="cuda")
    am.amulet_quantize_fp8_blocks(x, q, s)
    (bytes_q, q2), (store, s2) = matrices(layout, G, M, K, torch.float8_e4m3fn), matrices(layout, G, 2, 3, F32)
    am.amulet_quantize_fp8_blocks(x, q2, s2)
    assert torch.equal(q2.float(), q.float()) and torch.equal(s2, s)
    s2.fill_(7.0)
    assert (store == 7).all()
    q2.view(torch.uint8).copy_(torch.full(q2.shape, 7.0, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8))
    assert (bytes_q.float() == 7).all()


@pytest.mark.parametrize("trans_b", [False, True])
def test_8_bit_rows_far_apart(am, trans_b):
    """Rows of 8-bit operands at the longest pitch: the same as of rows side by side."""
    M, N, K, pitch = 130, 200, 150, 16711679
    g = gen(31)
    A, sa, B, sb = fp8_operands(g, M, K, (1, N, K) if trans_b else (1, K, N))
    R, far = torch.full((M, N), math.nan, device="cuda"), torch.full((M, N), math.nan, device="cuda")
    am.amulet_mm_fp8(A, sa, B[0], sb[0], R, trans_b=trans_b)

    def apart(x):
        y = torch.empty((x.shape[0] - 1) * pitch + x.shape[1], dtype=torch.uint8, device="cuda").as_strided(x.shape, (pitch, 1))
        y.copy_(x.view(torch.uint8))
        return y.view(torch.float8_e4m3fn)
    am.amulet_mm_fp8(apart(A), sa, apart(B[0]), sb[0], far, trans_b=trans_b)
    assert torch.equal(far, R)


def test_gradients_of_large_matrices(am):
    """128 matrices of 8192 x 8192, 17 GB: one group has all the rows, the last; the others' are zeros."""
    G, K, M = 128, 8192, 70
    g = gen(6)
    A, D = normal(g, M, K, dtype=BF16), normal(g, M, K, dtype=BF16)
    R = torch.full((G, K, K), 7.0, dtype=BF16, device="cuda")
    am.amulet_grouped_mm_wgrad(A, D, i32([0] * G + [M]), R)
    assert not R[:-1].any()
    a, d = A.double(), D.double()
    within(R[-1], a.t().contiguous() @ d, 2 * (M + 8) * 2.0 ** -24 * (a.abs().t().contiguous() @ d.abs()), "dB")


def test_a_large_quantisation(am):
    """2^20 rows of 16384: 34 GB of values, 2^34 of them; the last rows as alone."""
    M, K = 1 << 20, 1 << 14
    x = torch.zeros(M, K, dtype=BF16, device="cuda")
    x[-40:] = normal(gen(4), 40, K, dtype=BF16)
    q, s = torch.empty(M, K, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.full((K // 128, M), math.nan, device="cuda")
    am.amulet_quantize_fp8(x, q, s)
    q2, s2 = torch.empty(40, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(K // 128, 40, device="cuda")
    am.amulet_quantize_fp8(x[-40:].contiguous(), q2, s2)
    assert torch.equal(q[-40:].float(), q2.float()) and torch.equal(s[:, -40:], s2)
    assert (s[:, :-40] == 2.0 ** -126).all() and not q[:-40].view(torch.uint8).any()


def cancelling(g, M, N, K):
    """8-bit operands whose sums cancel: two products of 2^16 in every 128 k, one of each sign, and the others 2^-20 to 2^-18 of them.  In
    any order a block's partial sums are multiples of 2^-4 and at most 2^16 + 32, and up to 11 blocks' sums multiples of 2^-6
    and less than 2^11: fp32 holds them all."""
    f8 = torch.float8_e4m3fn
    a = torch.where(torch.empty(M, K, device="cuda").uniform_(generator=g) < 0.5, 0.25, 0.5)
    b = torch.where(torch.empty(K, N, device="cuda").uniform_(generator=g) < 0.5, 0.25, 0.5)
    for k in range(0, K - 1, 128):
        a[:, k:k + 2], b[k], b[k + 1] = 256.0, 256.0, -256.0
    sa = torch.exp2(torch.randint(-1, 2, ((K + 127) // 128, M), generator=g, device="cuda").float())
    sb = torch.exp2(torch.randint(-1, 2, (1, (K + 127) // 128, (N + 127) // 128), generator=g, device="cuda").float())
    return a.to(f8), sa, b[None].to(f8), sb


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 40, 128), (16, 8200, 256), (61, 200, 500), (300, 260, 136), (300, 129, 1321), (4096, 4000, 200), (256, 4096, 1024), (2048, 1024, 256)])
def test_8_bit_products_with_results_of_32_bits_drop_nothing(am, M, N, K, trans_b):
    """K products of two e4m3 values, each exact in 32 bits, and one scale of each 128: within what an fp32 sum of them may be off; and
    exact where fp32 holds every partial sum, however small beside the largest product."""
    print("8 bits, 32-bit results", M, N, K, trans_b, flush=True)
    g = gen(N + K)
    for random in (True, False):
        A, sa, B, sb = fp8_operands(g, M, K, (1, K, N)) if random else cancelling(g, M, N, K)
        av = A.double() * sa.t().double().repeat_interleave(128, 1)[:, :K]
        bv = B.double() * sb.double().repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 2)[:, :, :N]
        want, S = ref_rows(av, bv, [0, M], M, None, False)
        if trans_b:
            B, sb = B.transpose(1, 2).contiguous(), sb.transpose(1, 2).contiguous()
        R = torch.full((M, N), math.nan, device="cuda")
        am.amulet_mm_fp8(A, sa, B[0], sb[0], R, trans_b=trans_b)
        within(R, want, 2 * (K + sa.shape[0] + 8) * 2.0 ** -24 * S if random else torch.zeros_like(S), "R")


# sizes that the middle tile of the sums takes, with and without ranges of rows, and the largest one's ranges
@pytest.mark.parametrize("trans_r", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (FP16, FP16)])
@pytest.mark.parametrize("sizes,N,K,tokens,space,kernel", [
    ([400, 0, 505, 700], 1289, 1283, 0, 0, "128x128"), ([400, 0, 505, 700], 1289, 1283, 300, 0, "128x128"), ([64, 128, 1100, 13], 1296, 1288, 0, 0, "128x128"),
    ([5003, 3997], 1030, 1037, 0, 1 << 28, "128x128"), ([5003, 3997], 1030, 1037, 777, 1 << 28, "128x128"), ([12291], 5463, 672, 0, 1 << 28, "256x256"), ([12291], 5463, 672, 999, 1 << 28, "256x256")])
def test_gradients_by_the_larger_tiles(am, sizes, N, K, tokens, space, kernel, dtype, out, trans_r):
    print("gradients", kernel, sizes, N, K, tokens, space, dtype, out, trans_r, flush=True)
    g = gen(N + 7 * K)
    M, G = sum(sizes) + 5, len(sizes)
    at = offsets_of(sizes, 3)
    A, D = normal(g, tokens or M, K, dtype=dtype, pad=1), normal(g, M, N, dtype=dtype, shift=1)
    rows = torch.randint(-1, tokens + 1, (M,), generator=g, device="cuda", dtype=torch.int32) if tokens else None
    R = torch.full((G, N, K) if trans_r else (G, K, N), math.nan, dtype=out, device="cuda")
    ws = torch.full((space // 4,), math.nan, device="cuda") if space else None
    am.amulet_grouped_mm_wgrad(A, D, i32(at), R, ws, rows=rows, trans_r=trans_r)
    ran = am.amulet_recent_kernel()
    assert ran.split()[0] == "grouped_mm_wgrad_" + kernel and ("parts" in ran) == (space > 0)
    for e, (i, j) in enumerate(zip(at, at[1:])):
        a, d = A[i:j].double() if rows is None else A.double()[rows[i:j].clamp(0, tokens - 1).long()], D[i:j].double()
        if rows is not None:
            a[(rows[i:j] < 0) | (rows[i:j] >= tokens)] = 0
        w, s = a.t().contiguous() @ d, a.abs().t().contiguous() @ d.abs()
        within(R[e], w.t() if trans_r else w, 2 * (max(sizes) + 8) * 2.0 ** -24 * (s.t() if trans_r else s), "dB")
    again = torch.empty_like(R)
    am.amulet_grouped_mm_wgrad(A, D, i32(at), again, ws, rows=rows, trans_r=trans_r)
    assert torch.equal(R, again)


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("tokens", [0, 500])
def test_8_bit_products_of_many_matrices_with_some_rows_each(am, tokens, out, trans_b):
    g = gen(tokens + 1)
    sizes, N, K = [50, 64, 37, 0, 33, 64, 65, 49, 1, 63, 50, 60, 48, 51, 52, 70] * 2, 2003, 343
    M, G, at = sum(sizes), len(sizes), offsets_of(sizes)
    A, sa, B, sb = fp8_operands(g, tokens or M, K, (G, N, K) if trans_b else (G, K, N), pad=1)
    rows = torch.randint(-1, tokens + 1, (M,), generator=g, device="cuda", dtype=torch.int32) if tokens else None
    R = torch.full((M, N), math.nan, dtype=out, device="cuda")
    am.amulet_grouped_mm_fp8(A, sa, B, sb, i32(at), R, rows=rows, trans_b=trans_b)
    assert am.amulet_recent_kernel().split()[0] == "mm_fp8_64x128"
    check_fp8(R, A, sa, B, sb, at, rows, trans_b)


@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("sizes,N,K", [([5, 0, 9], 40, 72), ([300, 200, 100], 264, 200), ([2100, 1000, 1000], 4000, 136)])
def test_matrices_further_apart_and_shared(am, sizes, N, K, trans_b):
    """Every other matrix of a tensor, one matrix for all groups, and matrices whose rows lie in turn."""
    print("matrices apart", sizes, N, K, trans_b, flush=True)
    g = gen(N + K)
    M, G, at = sum(sizes), len(sizes), offsets_of(sizes)
    A = normal(g, M, K, dtype=BF16)
    shape = (N, K) if trans_b else (K, N)
    many = normal(g, 2 * G, *shape, dtype=BF16)
    turn = normal(g, shape[0], G, shape[1], dtype=BF16).permute(1, 0, 2)
    for B in (many[::2], many[1:2].expand(G, *shape), turn):
        R = torch.full((M, N), math.nan, dtype=BF16, device="cuda")
        am.amulet_grouped_mm(A, B, i32(at), R, trans_b=trans_b)
        want, S = ref_rows(A, B, at, M, None, trans_b)
        within(R, want, 2 * (K + 8) * 2.0 ** -24 * S, "R")
    A8, sa, B8, sb = fp8_operands(g, M, K, (2 * G,) + shape)
    R, packed = torch.full((M, N), math.nan, device="cuda"), torch.full((M, N), math.nan, device="cuda")
    am.amulet_grouped_mm_fp8(A8, sa, B8[::2], sb[::2], i32(at), R, trans_b=trans_b)
    am.amulet_grouped_mm_fp8(A8, sa, B8.view(torch.uint8)[::2].contiguous().view(torch.float8_e4m3fn), sb[::2].contiguous(), i32(at), packed, trans_b=trans_b)
    assert torch.equal(R, packed)
    check_fp8(R, A8, sa, B8[::2], sb[::2], at, None, trans_b)


@pytest.mark.parametrize("at", [[0, 70, 30, 90], [90, 60, 30, 0], [100, 0, 100, 0], [-7, 200, -9, 50], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 5]])
@pytest.mark.parametrize("N,K", [(40, 72), (300, 136)])
def test_offsets_that_do_not_ascend_touch_nothing_else(am, N, K, at):
    """What the results are is not said, but nothing beside them is written, and no value beside the operands reaches them."""
    print("offsets", at, N, K, flush=True)
    g = gen(N)
    M, G = 100, len(at) - 1
    A, B, D = normal(g, M, K, dtype=BF16, pad=2, shift=9), normal(g, G, K, N, dtype=BF16, pad=2, shift=9), normal(g, M, N, dtype=BF16, pad=2, shift=9)
    R = torch.full((50 + M, N + 4), 7.0, dtype=BF16, device="cuda")
    R[25:25 + M, 2:2 + N] = 0
    am.amulet_grouped_mm(A, B, i32(at), R[25:25 + M, 2:2 + N])
    assert torch.isfinite(R).all()
    R[25:25 + M, 2:2 + N] = 7.0
    assert (R == 7).all()
    for space in (None, torch.empty(1 << 22, dtype=torch.uint8, device="cuda")):
        W = torch.full((G + 2, K + 3, N + 4), 7.0, device="cuda")
        am.amulet_grouped_mm_wgrad(A, D, i32(at), W[1:1 + G, 1:1 + K, 2:2 + N], space)
        assert torch.isfinite(W).all()
        W[1:1 + G, 1:1 + K, 2:2 + N] = 7.0
        assert (W == 7).all()
