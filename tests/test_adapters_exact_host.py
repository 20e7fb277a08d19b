"""Problems of the low-rank adapters whose sums are whole numbers that fp32 holds, so that they come out the same in any order, and what a mistake
does to them (CPU only; the kernels are held to them in test_gpu_adapters_exact.py).

Ranks come in pairs whose T differ by a small number d, and R has the difference of one pair in each column: of T's some 20 bits only the last few are left, of
X W a few.  All sums lie below 2^20.  T is taken as three bf16 pieces; one of which nothing is left stands for 2^-30 of the one before, in up to two pieces
of two values of a column, and moves a sum by no more than a step of it each (2^-4 below 2^20): 0.25, and R's rounding (|R| < 256: 0.5 in bf16)."""
import pytest

torch = pytest.importorskip("torch")

F32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
LIMIT = 0.75


def generator(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def offsets_of(sizes):
    at = [0]
    for n in sizes:
        at.append(at[-1] + n)
    return at


def spans(at, which, G):
    return [(slice(i, j), a) for i, j, a in zip(at, at[1:], which) if j > i and 0 <= a < G]


def stored(x, transposed):
    return x.transpose(-1, -2).contiguous() if transposed else x.contiguous()


def mm_problem(seed, sizes, which, G, N, K, r, trans, spare=0, wide=False):
    """X, W, A, B as `trans` (of W, A, B) stores them, scales, offsets, adapters, in fp32.  wide: T below 2^10, B of 11 bits."""
    g = generator(seed)
    M = sum(sizes) + spare
    most = 3 if wide else max(1, min(127, 2 ** 20 // (256 * K) - 1))
    X = torch.randint(0, most + 1, (M, K), generator=g).float()
    X[:, K - 1] = 1
    A = torch.randint(0, max(1, 1000 // (3 * K)) + 1 if wide else 256, (G, K, r), generator=g).float()
    pairs = r // 2
    A[:, :, 1:2 * pairs:2] = A[:, :, 0:2 * pairs:2]
    i = torch.arange(pairs)
    d = 1 + (7 * torch.arange(G)[:, None] + 3 * i[None]) % 97
    A[:, K - 1, 0:2 * pairs:2] = (1 + d % 3 if wide else d).float()
    A[:, K - 1, 1:2 * pairs:2] = 0
    n = torch.arange(N)
    W = torch.zeros(K, N)
    W[torch.randint(0, K, (N,), generator=g), n] = torch.randint(-1, 2, (N,), generator=g).float()
    B = torch.zeros(G, r, N)
    if pairs:
        for a in range(G):
            at, sign = (n + 5 * a) % pairs, 1.0 - 2.0 * ((n // 3 + a) % 2)
            odd = (1025 + 2 * ((7 * n + a) % 511)).float() if wide else torch.ones(N)
            B[a, 2 * at, n] = sign * odd
            B[a, 2 * at + 1, n] = -sign * (odd - 2 if wide else odd)
    scales = 1.0 - 2.0 * (torch.arange(G) % 3 == 1).float()
    return X, stored(W, trans[0]), stored(A, trans[1]), stored(B, trans[2]), scales, offsets_of(sizes), (list(range(G)) if which is None else which)


def mm_answer(X, W, A, B, scales, at, which, trans, cut=None):
    """T and R in 64 bits, of T's values cut(T)."""
    x = X.double()
    w, a, b = (v.double().transpose(-1, -2) if t else v.double() for v, t in zip((W, A, B), trans))
    R, T = x @ w, torch.zeros(X.shape[0], a.shape[2], dtype=torch.float64, device=X.device)
    for rows, i in spans(at, which, a.shape[0]):
        T[rows] = float(scales[i]) * (x[rows] @ a[i])
        R[rows] += (T[rows] if cut is None else cut(T[rows])) @ b[i]
    return T, R


def pieces(x, n):
    """n bf16 pieces of values that fp32 holds, the last one rounded."""
    out, rest = torch.zeros_like(x), x.float()
    for p in range(n):
        first = rest.bfloat16().float() if p == n - 1 else (rest.view(torch.int32) & -65536).view(torch.float32)
        out, rest = out + first.double(), rest - first
    return out


def outer_problem(seed, sizes, which, G, N, r):
    """X of -1, 0 and 1 and T of whole numbers to 7, in fp32: sums of either sign, |R| a few thousand at most."""
    g = generator(seed)
    M = sum(sizes)
    X, T = torch.randint(-1, 2, (M, N), generator=g).float(), torch.randint(-7, 8, (M, r), generator=g).float()
    X[:, 0], T[:, 0] = 1, torch.where(torch.arange(M) % 2 == 0, 5.0, -4.0)      # (every row counts)
    return X, T, offsets_of(sizes), (list(range(G)) if which is None else which)


def outer_answer(X, T, at, which, G):
    R = torch.zeros(G, X.shape[1], T.shape[1], dtype=torch.float64, device=X.device)
    for rows, i in spans(at, which, G):
        R[i] += X[rows].double().t() @ T[rows].double()
    return R


def fine_problem(seed, sizes, which, G, N, r):
    """Rows in pairs, one times 1 and one times -1, whose T of 20 bits differ by a small number."""
    X, _, at, which = outer_problem(seed, sizes, which, G, N, r)
    M = X.shape[0]
    g = generator(seed + 1)
    T = torch.zeros(M, r)
    X = torch.zeros(M, N)
    for rows, _a in spans(at, which, G):
        at_pair = torch.arange(rows.start, rows.stop - 1, 2)
        few = at_pair[torch.randperm(len(at_pair), generator=g)[:6]]
        t = torch.randint(2 ** 19, 2 ** 20, (len(few), r), generator=g).float()
        d = torch.randint(1, 40, (len(few), r), generator=g).float()
        T[few], T[few + 1] = t, t - d
        sign = torch.randint(0, 2, (len(few), N), generator=g).float() * 2 - 1
        X[few], X[few + 1] = sign, -sign
    return X, T, at, which


def fine_limit(at, which, G, T):
    """What the sums of a fine_problem may be off by.  Each is a whole number below 2^11, but for the stand-ins (2^-10 of a T below 2^20 at most, some 2^-18 mostly), and all
    of its additions but those of T's first pieces are of values below 2^13, whose steps are 2^-10.  An addition in which a first piece takes part (below 2^20: a step of 2^-4) keeps no less
    than that step of the sum before it, whichever way it rounds; two such for each step of 32 rows that has any."""
    steps = [0] * G
    for rows, i in spans(at, which, G):
        steps[i] += sum(bool((T[k:min(k + 32, rows.stop)] != 0).any()) for k in range(rows.start, rows.stop, 32))
    return 0.25 + 2 * 2.0 ** -4 * max(steps)


@pytest.mark.parametrize("K,r,N", [(136, 16, 40), (520, 72, 96), (1032, 9, 30), (64, 128, 130)])
def test_mistakes_show(K, r, N):
    """Two pieces of T in place of three, another adapter's matrices, a neighbour's row."""
    sizes, which, G, trans = [20, 0, 9, 3], [1, 0, 2, -1], 3, (False, False, False)
    X, W, A, B, scales, at, who = mm_problem(K, sizes, which, G, N, K, r, trans, spare=2)
    T, R = mm_answer(X, W, A, B, scales, at, who, trans)
    assert float(T.abs().max()) < 2 ** 20 and float(R.abs().max()) < 256 and torch.equal(T, T.round())
    assert torch.equal(pieces(T, 3), T) and torch.equal(mm_answer(X, W, A, B, scales, at, who, trans, lambda t: pieces(t, 3))[1], R)
    rows = slice(0, 20)
    off = (mm_answer(X, W, A, B, scales, at, who, trans, lambda t: pieces(t, 2))[1] - R).abs()
    assert float((off[rows] > LIMIT).double().mean()) > 0.3
    for other in ([1, 0, 0, -1], [-1, 0, 2, -1], [1, 0, 2, 0]):
        off = (mm_answer(X, W, A, B, scales, at, other, trans)[1] - R).abs()
        assert (off > LIMIT).any()
    off = (mm_answer(X, W, A, B, scales, [0, 19, 20, 29, 32], who, trans)[1] - R).abs()       # (a row less)
    assert (off[19] > LIMIT).any()


def test_eleven_bits_of_b_show():
    sizes, G, N, K, r, trans = [40, 13], 2, 64, 32, 12, (True, True, True)
    X, W, A, B, scales, at, who = mm_problem(7, sizes, None, G, N, K, r, trans, wide=True)
    T, R = mm_answer(X, W, A, B, scales, at, who, trans)
    assert float(T.abs().max()) < 2 ** 10 and float(R.abs().max()) < 2 ** 22 and torch.equal(B.half().float(), B) and not torch.equal(B.bfloat16().float(), B)
    off = (mm_answer(X, W, A, B.bfloat16().float(), scales, at, who, trans)[1] - R).abs()
    assert float((off > 16).double().mean()) > 0.3


@pytest.mark.parametrize("sizes,which,G", [([4000], None, 1), ([20000, 100], None, 2), ([700, 31, 1, 300], [1, 0, 1, 1], 2), ([9] * 148, [i % 3 for i in range(148)], 3)])
def test_a_row_left_out_shows(sizes, which, G):
    X, T, at, who = outer_problem(3, sizes, which, G, 24, 8)
    R = outer_answer(X, T, at, who, G)
    for row in (0, 31, 32, sum(sizes) - 1, sum(sizes) // 2):
        less = T.clone()
        less[row] = 0
        assert float((outer_answer(X, less, at, who, G) - R).abs().max()) > LIMIT
    X, T, at, who = fine_problem(4, sizes, which, G, 24, 8)
    R = outer_answer(X, T, at, who, G)
    off = (outer_answer(X, pieces(T.double(), 2), at, who, G) - R).abs()
    assert float((off > fine_limit(at, who, G, T)).double().mean()) > 0.3 and torch.equal(pieces(T.double(), 3), T.double())
