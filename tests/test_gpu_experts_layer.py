"""The example layer, whose forward, backward and 8-bit passes run the mixture-of-experts operators together, against the
same layer in 64 bits; and the compiled marshalling of their calls against the Python one."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import experts_layer
    return experts_layer


def near(a, b, rel):
    return float((a.double() - b).norm()) <= rel * float(b.norm())


@pytest.mark.parametrize("T,width,hidden,E,k", [(1, 64, 96, 8, 2), (37, 72, 40, 5, 3), (300, 128, 200, 16, 4)])
def test_layer_against_64_bits(ex, T, width, hidden, E, k):
    print("layer", T, width, hidden, E, k, flush=True)
    layer = ex.Layer(width, hidden, E, k, seed=T)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    x = torch.empty(T, width, device="cuda").normal_(generator=g).bfloat16()
    dout = torch.empty(T, width, device="cuda").normal_(generator=g).bfloat16()
    out = layer.forward(x)
    dx, drouter, dw1, dw2 = layer.backward(dout)

    # the definition: every expert on every token, the chosen ones weighted
    p = {n: getattr(layer, n).double().cpu().requires_grad_() for n in ("router", "w1", "w2")}
    x64 = x.double().cpu().requires_grad_()
    logits = x64 @ p["router"]
    chosen = layer.chosen.long().cpu()
    w = torch.softmax(logits.gather(1, chosen), 1)
    y = torch.stack([torch.nn.functional.silu(x64 @ p["w1"][e]) @ p["w2"][e] for e in range(E)], 1)
    want = (w[:, :, None] * y.gather(1, chosen[:, :, None].expand(-1, -1, width))).sum(1)
    (want * dout.double().cpu()).sum().backward()
    # five roundings to bf16 (2^-8 each at most) lie on the longest way
    rel = 5 * 2.0 ** -8
    assert near(out.cpu(), want.detach(), rel)
    assert near(dx.cpu(), x64.grad, rel)
    for got, name in ((drouter, "router"), (dw1, "w1"), (dw2, "w2")):
        assert near(got.cpu(), p[name].grad, rel), name
    # the choice is by the logits themselves
    assert torch.equal(torch.sort(layer.logits, dim=1, descending=True, stable=True)[1][:, :k].int(), layer.chosen)
    layer.quantize()
    # (two operands of 2^-4 at most, twice: e4m3 has 4 significant bits)
    assert near(layer.forward_8bit(x).cpu(), want.detach(), 4 * 2.0 ** -4)


def test_example_learns(ex):
    losses, off = ex.main(tokens=256, width=128, hidden=128, experts=4, k=2, steps=6)
    assert losses[-1] < losses[0] and off < 4 * 2.0 ** -4


def test_compiled_marshalling_reads_what_the_python_one_reads(ex, monkeypatch):
    """Every call through both, on views and on a side stream: same results; what neither takes raises."""
    am = ex.am
    from paper_2305_08872_amd import binding
    assert binding._marshal is not None, "the compiled marshalling is not built"
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    T, E, k, K, N = 20, 6, 2, 40, 24

    def normal(*shape, dtype=torch.bfloat16):
        wide = torch.empty(*shape[:-1], shape[-1] + 3, device="cuda").normal_(generator=g).to(dtype)
        return wide[..., :shape[-1]]
    logits, x, B, D, up = normal(T, E, dtype=torch.float32), normal(T, K), normal(E, K, N), normal(T * k, N), normal(T, k, dtype=torch.float32).contiguous()
    i32 = dict(dtype=torch.int32, device="cuda")

    def all_calls(stream):
        o = {"e": torch.empty(T, k, **i32), "w": torch.empty(T, k, device="cuda"), "p": torch.empty(T, k, **i32), "t": torch.empty(T * k, **i32),
             "o": torch.empty(E + 1, **i32)}
        am.amulet_route(logits, o["e"], o["w"], o["p"], o["t"], o["o"], norm=False, stream=stream)
        o["dl"] = torch.empty(T, E + 1, device="cuda")[:, :E]
        am.amulet_route_grad(logits, o["e"], o["w"], up, o["dl"], norm=False, stream=stream)
        o["dl2"] = torch.empty(T, E, device="cuda")
        am.amulet_route_grad(None, o["e"], o["w"], up, o["dl2"], stream=stream)
        o["r"] = torch.empty(T * k, N + 2, device="cuda")[:, :N]
        am.amulet_grouped_mm(x, B, o["o"], o["r"], rows=o["t"], stream=stream)
        o["da"] = torch.empty(T * k, K, dtype=torch.bfloat16, device="cuda")
        am.amulet_grouped_mm(D, B, o["o"], o["da"], trans_b=True, stream=stream)
        o["dw"], o["dwt"] = torch.empty(E, K, N, device="cuda"), torch.empty(E, N, K, device="cuda")
        ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
        am.amulet_grouped_mm_wgrad(x, D, o["o"], o["dw"], ws, rows=o["t"], stream=stream)
        am.amulet_grouped_mm_wgrad(x, D, o["o"], o["dwt"], rows=o["t"], trans_r=True, stream=stream)
        o["c"], o["cx"] = torch.empty(T, N, dtype=torch.bfloat16, device="cuda"), torch.empty(T, K, dtype=torch.bfloat16, device="cuda")
        am.amulet_combine(D, o["w"], o["p"], o["c"], stream=stream)
        am.amulet_combine(o["da"], None, o["p"], o["cx"], stream=stream)
        o["dy"], o["dcw"] = torch.zeros(T * k, N, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, device="cuda")
        am.amulet_combine_grad(D, o["w"], o["p"], o["c"], o["dy"], o["dcw"], stream=stream)
        am.amulet_combine_grad(None, None, o["p"], o["c"], o["dy"], stream=stream)
        q, s = torch.empty(T, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(1, T, device="cuda")
        qb, sb = torch.empty(E, K, N, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(E, 1, 1, device="cuda")
        am.amulet_quantize_fp8(x, q, s, stream=stream)
        am.amulet_quantize_fp8_blocks(B, qb, sb, stream=stream)
        o["q"], o["s"], o["qb"], o["sb"] = q.float(), s, qb.float(), sb
        o["f"], o["fd"] = torch.empty(T * k, N, device="cuda"), torch.empty(T, N, dtype=torch.float16, device="cuda")
        am.amulet_grouped_mm_fp8(q, s, qb, sb, o["o"], o["f"], rows=o["t"], stream=stream)
        am.amulet_mm_fp8(q, s, qb[2], sb[2], o["fd"], stream=stream)
        return o
    side = torch.cuda.Stream()
    results = []
    for stream in (None, side, side.cuda_stream):
        for compiled in (True, False):
            with monkeypatch.context() as m:
                if not compiled:
                    m.setattr(binding, "_marshal", None)
                torch.cuda.synchronize()
                with torch.cuda.stream(side if stream is not None else torch.cuda.current_stream()):
                    results.append(all_calls(stream))
                torch.cuda.synchronize()
    for other in results[1:]:
        for name, v in results[0].items():
            assert torch.equal(v, other[name]), name
    for compiled in (True, False):
        with monkeypatch.context() as m:
            if not compiled:
                m.setattr(binding, "_marshal", None)
            o = results[0]
            for bad in (lambda: am.amulet_grouped_mm(x.float().half(), B, o["o"], o["r"], rows=o["t"]), lambda: am.amulet_grouped_mm(x, B, o["o"], o["r"]),
                        lambda: am.amulet_grouped_mm(x, B, o["o"].long(), o["r"], rows=o["t"]), lambda: am.amulet_grouped_mm(x, B, o["o"][:-1], o["r"], rows=o["t"]),
                        lambda: am.amulet_grouped_mm(x, B, o["o"], o["r"], rows=o["t"][:-1]), lambda: am.amulet_grouped_mm(x, B, o["o"], o["da"], rows=o["t"]),
                        lambda: am.amulet_grouped_mm(x.cpu(), B, o["o"], o["r"], rows=o["t"]), lambda: am.amulet_route(logits, o["e"][:-1], o["w"], o["p"], o["t"], o["o"]),
                        lambda: am.amulet_route(logits.double(), o["e"], o["w"], o["p"], o["t"], o["o"]), lambda: am.amulet_combine(D.half(), o["w"], o["p"], o["c"]),
                        lambda: am.amulet_combine(D, o["w"], o["p"][:-1], o["c"]), lambda: am.amulet_quantize_fp8(x, o["da"], o["s"]),
                        lambda: am.amulet_mm_fp8(o["q"], o["s"], o["qb"][0], o["sb"][0], o["fd"])):
                with pytest.raises(ValueError):
                    bad()
            with pytest.raises(am.AmuletError):      # R of neither the operands' type nor fp32
                am.amulet_grouped_mm(x, B, o["o"], o["fd"].repeat(k, 1), rows=o["t"])
            many = torch.empty(100, E, device="cuda")
            with pytest.raises(am.AmuletError):      # no workspace
                am.amulet_route(many, torch.empty(100, k, **i32), torch.empty(100, k, device="cuda"), torch.empty(100, k, **i32), torch.empty(100 * k, **i32), o["o"])
