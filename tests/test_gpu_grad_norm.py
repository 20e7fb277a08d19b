"""The norm of several tensors and their clipping against 64 bits.

Squares are summed in fp64: the norm is within one rounding to fp32 (2^-24) of the exact one, but for the sum's own 2^-40.  The factor
max_norm / norm has the norm's rounding and its own, the product one more, and the result is rounded once to its type."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, FP16: 2.0 ** -11}
LEAST = {F32: 2.0 ** -149, BF16: 2.0 ** -134, FP16: 2.0 ** -25}


@pytest.fixture(scope="module")
def am():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2305_08872_amd as am
    am.load_library()
    return am


def make(counts, seed=0, types=(F32, BF16, FP16), shift=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for i, n in enumerate(counts):
        x = torch.empty(n + shift + 3, device="cuda").normal_(0, scale, generator=g).to(types[i % len(types)])
        x[:shift], x[shift + n:] = math.nan, math.nan
        out.append(x[shift:shift + n])
    return out


def exact_norm(grads):
    return math.sqrt(sum(float((x.double() ** 2).sum()) for x in grads))


def workspace(am, n):
    return torch.empty(max(1, am.amulet_grad_norm_workspace_bytes(n)), dtype=torch.uint8, device="cuda")


def check_norm(got, want):
    assert abs(float(got) - want) <= (2.0 ** -24 + 2.0 ** -40) * want, (float(got), want)


def check_clipped(outs, grads, want, most):
    f = min(1.0, most / want) if want > 0 else 1.0
    for o, x in zip(outs, grads):
        if f == 1.0:
            assert torch.equal(o, x)
            continue
        exact = x.double() * f
        limit = (3 * 2.0 ** -24 + HALF_ULP[x.dtype] + 2.0 ** -30) * exact.abs() + LEAST[x.dtype]
        assert ((o.double() - exact).abs() <= limit).all()


COUNTS = [[1], [5, 0, 3], [8192], [8191, 8193, 1], [1 << 20, 17, 4096], [100003, 9, 8192 * 3], [64] * 180, [1000 + i for i in range(181)],
          [3 * i for i in range(400)]]


@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("types", [(F32,), (BF16,), (FP16,), (F32, BF16, FP16)])
@pytest.mark.parametrize("counts", COUNTS)
def test_norm_and_clip(am, counts, types, shift):
    print("norm", counts[:6], len(counts), types, shift, flush=True)
    grads = make(counts, len(counts), types, shift)
    want, n = exact_norm(grads), len(counts)
    norm, ws = torch.full((1,), math.nan, device="cuda"), workspace(am, n)
    am.amulet_grad_norm(grads, norm, ws)
    check_norm(norm, want)
    for most in (0.37 * want, 1.5 * want, math.inf, 0.0):
        whole = [torch.full((x.numel() + 4,), 5.0, dtype=x.dtype, device="cuda") for x in grads]
        outs = [w[2:2 + x.numel()] for w, x in zip(whole, grads)]
        before = [x.clone() for x in grads]
        again = torch.full((1,), math.nan, device="cuda")
        am.amulet_grad_norm_clip(grads, most, again, ws, outs=outs)
        assert torch.equal(norm, again) and all(torch.equal(x, y) for x, y in zip(grads, before))
        check_clipped(outs, grads, want, most)
        assert all((w[:2] == 5).all() and (w[-2:] == 5).all() for w in whole)
        # in two calls the same bits, and in place
        two = [torch.empty_like(x) for x in grads]
        am.amulet_grad_clip(grads, most, norm, outs=two)
        inplace = [x.clone() for x in grads]
        am.amulet_grad_norm_clip(inplace, most, again, ws)
        assert all(torch.equal(x, y) for x, y in zip(outs, two)) and all(torch.equal(x, y) for x, y in zip(outs, inplace))


def test_more_tensors_than_workgroups_add_up_for_themselves(am):
    counts = [9 * 8192 + i for i in range(1000)]
    grads = make(counts, 3, (BF16, F32))
    want = exact_norm(grads)
    norm = torch.empty(1, device="cuda")
    am.amulet_grad_norm_clip(grads, 0.5 * want, norm, workspace(am, 1000), outs=(outs := [torch.empty_like(x) for x in grads]))
    check_norm(norm, want)
    check_clipped(outs, grads, want, 0.5 * want)


def test_large_and_small_values(am):
    """Squares past fp32's range either way, and a small tensor beside a large one."""
    for scale in (1e25, 1e-25, 1e30):
        grads = make([5000, 77], 4, (F32, BF16), scale=scale)
        norm = torch.empty(1, device="cuda")
        am.amulet_grad_norm(grads, norm, workspace(am, 2))
        check_norm(norm, exact_norm(grads))
    tiny = torch.full((100,), 2.0 ** -149, device="cuda")       # the least fp32 value
    am.amulet_grad_norm([tiny], norm, workspace(am, 1))
    assert float(norm) == 10 * 2.0 ** -149
    am.amulet_grad_norm([torch.zeros(10, device="cuda")], norm, workspace(am, 1))
    assert float(norm) == 0.0


def test_norms_that_are_no_numbers_change_nothing(am):
    for bad in (math.nan, math.inf, -math.inf):
        grads = make([3000, 40], 5)
        grads[1][7] = bad
        before = [x.clone() for x in grads]
        norm, ws = torch.zeros(1, device="cuda"), workspace(am, 2)
        outs = [torch.empty_like(x) for x in grads]
        am.amulet_grad_norm_clip(grads, 1.0, norm, ws, outs=outs)
        assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
        assert all(torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0)) for x, y in zip(outs, before))
        am.amulet_grad_norm_clip(grads, 1.0, norm, ws)
        am.amulet_grad_clip(grads, 1.0, norm)
        assert all(torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0)) for x, y in zip(grads, before))
    # finite values whose norm fp32 does not hold
    grads = [torch.full((10000,), 3e38, device="cuda")]
    am.amulet_grad_norm_clip(grads, 1.0, norm, workspace(am, 1))
    assert float(norm) == math.inf and (grads[0] == 3e38).all()


def test_lists_without_values(am):
    norm, ws = torch.full((1,), math.nan, device="cuda"), workspace(am, 1)
    empty = torch.empty(0, device="cuda")
    for grads in ([], [empty], [empty] * 200):
        norm.fill_(math.nan)
        am.amulet_grad_norm(grads, norm, workspace(am, len(grads)))
        assert float(norm) == 0.0
        norm.fill_(math.nan)
        am.amulet_grad_norm_clip(grads, 1.0, norm, workspace(am, len(grads)))
        assert float(norm) == 0.0
        am.amulet_grad_clip(grads, 1.0, norm)
    del ws


def test_other_layouts_and_parameters(am):
    """Matrices, transposed ones, parameters' gradients; a tensor with gaps is refused."""
    p = torch.nn.Parameter(torch.zeros(30, 40, device="cuda"))
    p.grad = torch.randn(30, 40, device="cuda")
    t = torch.randn(50, 60, device="cuda").bfloat16().t()
    grads = [p.grad, t, torch.randn(2, 3, 4, device="cuda").permute(2, 0, 1)]
    want, before = exact_norm(grads), [x.clone() for x in grads]
    norm, ws = torch.empty(1, device="cuda"), workspace(am, 3)
    am.amulet_grad_norm_clip(grads, 1.0, norm, ws)
    check_norm(norm, want)
    check_clipped(grads, before, want, 1.0)
    for bad in (torch.randn(10, 12, device="cuda")[:, :7], torch.randn(5, 1, device="cuda").expand(5, 4), torch.zeros(4, dtype=torch.int32, device="cuda"),
                torch.zeros(4), torch.zeros(4, dtype=torch.float64, device="cuda")):
        with pytest.raises(ValueError):
            am.amulet_grad_norm([grads[0], bad], norm, ws)
    with pytest.raises(ValueError):
        am.amulet_grad_norm_clip(grads, 1.0, norm, ws, outs=[torch.empty_like(x) for x in grads[:2]])
    with pytest.raises(ValueError):
        am.amulet_grad_norm_clip(grads[:1], 1.0, norm, ws, outs=[torch.empty(1200, device="cuda")])
    with pytest.raises(am.AmuletError):
        am.amulet_grad_norm_clip(grads, -1.0, norm, ws)
    with pytest.raises(am.AmuletError):
        am.amulet_grad_norm(grads, norm, ws[:8])


def test_a_captured_clip_replays(am):
    grads = make([5000, 8192 * 5, 33], 6)
    start = [x.clone() for x in grads]
    norm, ws = torch.empty(1, device="cuda"), workspace(am, 3)
    outs = [torch.empty_like(x) for x in grads]
    graph = torch.cuda.CUDAGraph()
    am.amulet_grad_norm_clip(grads, 2.0, norm, ws, outs=outs)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        am.amulet_grad_norm_clip(grads, 2.0, norm, ws, outs=outs)
    for n in range(4):
        for x, y in zip(grads, start):
            x.copy_(y * (n + 0.5))
        norm.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        want = exact_norm(grads)
        check_norm(norm, want)
        check_clipped(outs, grads, want, 2.0)


def test_a_tensor_of_more_than_4_gib(am):
    x = torch.zeros((1 << 31) + 12345, dtype=BF16, device="cuda")
    x[-1], x[0], x[(1 << 31) + 5] = 3.0, 4.0, 12.0
    norm = torch.empty(1, device="cuda")
    am.amulet_grad_norm_clip([x], 6.5, norm, workspace(am, 1))
    assert float(norm) == 13.0 and float(x[-1]) == 1.5 and float(x[0]) == 2.0 and float(x[(1 << 31) + 5]) == 6.0
    assert int((x != 0).sum()) == 3
