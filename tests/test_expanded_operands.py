"""Tensors whose rows lie on one another (torch's expand(): the gradient of a sum is one), of one column too, where a row's pitch of nothing could
be taken for that of a column: refused, not read as rows one behind the other."""
import pytest

torch = pytest.importorskip("torch")

from paper_2305_08872_amd import binding  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


class OnTheGpu:
    """What the binding asks of a tensor, of one that lies on the CPU."""
    is_cuda = True

    def __init__(self, t):
        self.t, self.dtype, self.shape = t, t.dtype, t.shape

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.mark.parametrize("rows,cols,pitch", [(1, 1, 1), (1, 5, 5), (4, 5, 5), (4, 1, 1), (0, 3, 3), (3, 0, 1), (0, 0, 1)])
def test_pitches_of_ordinary_tensors(rows, cols, pitch):
    assert binding._mat(OnTheGpu(torch.zeros(rows, cols)), F32, "X")[1:] == (rows, cols, pitch)
    assert binding._groups(OnTheGpu(torch.zeros(2, rows, cols)), F32, "A")[1:5] == (2, rows, cols, pitch)


def test_expanded_rows_keep_a_pitch_of_nothing():
    for cols in (1, 3):
        x = torch.zeros(1, cols).expand(5, cols)
        assert binding._mat(OnTheGpu(x), F32, "X")[1:] == (5, cols, 0)
        assert binding._groups(OnTheGpu(x[None].expand(2, 5, cols)), F32, "A")[1:] == (2, 5, cols, 0, 0)
    assert binding._mat(OnTheGpu(torch.zeros(1, 3).expand(1, 3)), F32, "X")[3] == 3


@pytest.mark.gpu
def test_calls_refuse_them():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2305_08872_amd as am
    am.load_library()
    bf = dict(dtype=BF16, device="cuda")
    M, one = 300, torch.ones(1, 1, **bf)
    off, t, y = torch.tensor([0, 100, M], dtype=torch.int32, device="cuda"), torch.zeros(M, 1, device="cuda"), torch.zeros(M, 1, **bf)
    w, a = torch.ones(1, 1, **bf), torch.ones(2, 1, 1, **bf)
    calls = [lambda: am.amulet_adapters_mm(one.expand(M, 1), w, a, a, off, t, y), lambda: am.amulet_adapters_mm(y, w, a, a, off, torch.zeros(1, 1, device="cuda").expand(M, 1), y),
             lambda: am.amulet_adapters_mm(y, w, a, a, off, t, one.expand(M, 1)), lambda: am.amulet_adapters_wgrad(one.expand(M, 1), t, off, torch.zeros(2, 1, 1, device="cuda")),
             lambda: am.amulet_adapters_mm(torch.zeros(M, 8, **bf), torch.zeros(8, 1, **bf), torch.ones(1, 1, 1, **bf).expand(2, 8, 1), a, off, t, y),
             lambda: am.amulet_grouped_mm(one.expand(M, 1), a, off, y), lambda: am.amulet_grouped_mm(y, a, off, one.expand(M, 1)),
             lambda: am.amulet_mmlike_f32(0, torch.ones(1, 1, device="cuda").expand(M, 1), torch.ones(1, 5, device="cuda"), None, torch.zeros(M, 5, device="cuda"))]
    for plain in (False, True):
        marshal, binding._marshal = binding._marshal, None if plain else binding._marshal
        try:
            for n, call in enumerate(calls):
                with pytest.raises(am.AmuletError) as e:
                    call()
                assert e.value.code == -4, n
        finally:
            binding._marshal = marshal
