"""The operators that a mixture-of-experts layer is made of, as cases that can be timed.

  router           for every token the k experts with the highest logits, their weights, and the rows of all
                   (token, expert) pairs in order of expert (route); the weighted sum that brings the experts'
                   rows back to their tokens (combine); both with their gradients
  grouped product  R[i] = A[row(i)] B[g] for the rows i of every expert g, 16-bit operands, with both gradients
  fp8 product      the same, dense or by expert, of 8-bit operands with one scale for each block of 128, and the
                   quantiser that makes them

  own               whether run() calls the library or computes the plain form
  listed()          the cases
  draw(rng)         one more case of the same ranges
  prepare(case, s)  what a program has in hand before the call, from seed s
  run(state)        one pass; returns the outputs
  work(case)        bytes and operations that no implementation can do without
  exact(case, s)    run()'s outputs from the definition in 64 bits
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
FP8_MOST = 448.0            # the largest value of an e4m3 number
SCALE_LEAST = 2.0 ** -126   # of a block of zeros


def listed():
    return [
        # the router of a layer that decodes eight sequences: latency
        dict(name="route_decode", op="route", T=8, E=64, k=6, norm=True, type="fp32", masked=0.0, grad=False),
        # a training step's router over 16384 tokens, forward and backward, some experts and some tokens masked
        dict(name="route_train", op="route", T=16384, E=128, k=8, norm=False, type="fp32", masked=0.02, grad=True),
        # the experts' rows of eight decoded tokens brought back
        dict(name="combine_decode", op="combine", T=8, k=6, H=4096, type="bf16", masked=0.0, grad=False),
        # ... of a training step, forward and backward, with pairs that were dropped
        dict(name="combine_train", op="combine", T=16384, k=8, H=2048, type="bf16", masked=0.02, grad=True),
        # eight decoded tokens through six of 64 experts each: the weights' bytes count
        dict(name="grouped_decode", op="grouped", M=48, G=64, N=2048, K=2048, type="bf16", out="bf16", trans_b=True, tokens=8, spare=0, grad=False),
        # 8192 prompt tokens through four of 32 experts each, gathered from the tokens' rows: the largest product
        dict(name="grouped_prompt", op="grouped", M=32768, G=32, N=4096, K=4096, type="bf16", out="bf16", trans_b=True, tokens=8192, spare=0, grad=False),
        # sizes as they fall, fp16, sums kept in 32 bits, rows that belong to no expert
        dict(name="grouped_odd", op="grouped", M=3001, G=7, N=1501, K=1003, type="fp16", out="fp32", trans_b=False, tokens=0, spare=40, grad=False),
        # the backward pass of a layer's product: the gradients of the rows and of every expert's weights
        dict(name="grouped_grad", op="grouped", M=16384, G=16, N=4096, K=2048, type="bf16", out="bf16", trans_b=True, tokens=0, spare=0, grad=True),
        # a prompt's activations on their way into an fp8 product
        dict(name="quantize_rows", op="quantize", G=1, M=16384, K=4096, type="bf16", rows=1),
        # eight decoded tokens through a dense fp8 layer
        dict(name="fp8_decode", op="fp8", M=8, G=0, N=8192, K=4096, out="bf16", trans_b=True, tokens=0),
        # prompt tokens through fp8 experts
        dict(name="fp8_prompt", op="fp8", M=32768, G=16, N=4096, K=4096, out="bf16", trans_b=True, tokens=8192),
        # the gradient of the rows, the weights read the other way, sizes that end inside blocks
        dict(name="fp8_odd", op="fp8", M=1777, G=5, N=1368, K=2504, out="fp32", trans_b=False, tokens=0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """The width of a layer: mostly whole 64s or 8s, one in six as it falls."""
    n, kind = _log(rng, low, high), rng.random()
    n = max(64, n // 64 * 64) if kind < 0.6 else max(8, n // 8 * 8) if kind < 0.84 else n
    return n if n != 3072 else 3008   # (not a width that this repository has)


def draw(rng):
    """One to 32768 rows, 1 to 128 experts, widths of 64 to 4096, every type and direction; no dearer than the
    largest listed case of its kind."""
    op = rng.choice(["route", "combine", "grouped", "grouped", "grouped", "quantize", "fp8", "fp8"])
    if op == "route":
        E = _log(rng, 4, 256)
        return dict(op=op, T=_log(rng, 1, 16384), E=E, k=rng.randint(1, min(8, E)), norm=rng.random() < 0.5,
                    type=rng.choice(["fp32", "fp32", "bf16", "fp16"]), masked=rng.choice([0.0, 0.02, 0.2]), grad=rng.random() < 0.5)
    if op == "combine":
        return dict(op=op, T=_log(rng, 1, 16384), k=rng.randint(1, 8), H=_width(rng, 64, 2048),
                    type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), masked=rng.choice([0.0, 0.02, 0.2]), grad=rng.random() < 0.5)
    if op == "quantize":
        whole = rng.random() < 0.3
        G, M = (rng.randint(1, 8), _width(rng, 64, 2048)) if whole else (1, _log(rng, 1, 16384))
        return dict(op=op, G=G, M=M, K=_width(rng, 64, 4096), type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), rows=128 if whole else 1)
    grad = op == "grouped" and rng.random() < 0.4
    G = _log(rng, 1, 128)
    while True:
        M, N, K = _log(rng, 1, 32768), _width(rng, 64, 4096), _width(rng, 64, 4096)
        if M * N * K <= (2 ** 37 if grad else 2 ** 38) and G * N * K <= 2 ** 29:
            break
    tokens = 0 if rng.random() < 0.5 else max(1, M // rng.randint(1, 8))
    if op == "fp8":
        return dict(op=op, M=M, G=0 if rng.random() < 0.4 else G, N=N, K=K, out=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    trans_b=rng.random() < 0.6, tokens=tokens)
    kind = rng.choice(["bf16", "bf16", "fp16"])
    return dict(op=op, M=M, G=G, N=N, K=K, type=kind, out=rng.choice([kind, "fp32"]), trans_b=rng.random() < 0.5, tokens=tokens,
                spare=rng.choice([0, 0, M // 50]), grad=grad)


# ------------------------------------------------------------------------------------------------ inputs

def _shares(G):
    """How often each of G experts is chosen: unevenly, as a trained router does."""
    p = [(1 + g) ** -0.25 for g in range(G)]
    return [x / sum(p) for x in p]


def _sizes(M, G, seed):
    rng = random.Random(seed * 1000003 + M * 31 + G)
    shares = _shares(G)
    rng.shuffle(shares)
    n = [0] * G
    for g in rng.choices(range(G), shares, k=M):
        n[g] += 1
    return n


def _offsets(sizes):
    at = [0]
    for n in sizes:
        at.append(at[-1] + n)
    return at


def _by_expert(experts, E):
    """place, tokens and offsets of chosen experts (-1: none): rows in order of expert, then of token."""
    T, k = experts.shape
    key = torch.where(experts < 0, E, experts).reshape(-1).long()
    keys, order = torch.sort(key, stable=True)
    row = torch.empty_like(order)
    row[order] = torch.arange(T * k, device=key.device)
    place = torch.where(key < E, row, -1).reshape(T, k).int()
    tokens = torch.where(keys < E, order // k, -1).int()
    offsets = torch.searchsorted(keys, torch.arange(E + 1, device=key.device)).int()
    return place, tokens, offsets


def _blocks(x, rows):
    """x (G x M x K) in 32 bits as G x RB x rows x KB x 128, the edges filled with zeros."""
    G, M, K = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -K % 128, 0, -M % rows))
    return x.view(G, x.shape[1] // rows, rows, x.shape[2] // 128, 128)


def _quantized(x, rows):
    """(values in e4m3, scales) of x, G x M x K: a scale for each `rows` x 128 block, G x RB x KB."""
    G, M, K = x.shape
    b = _blocks(x, rows)
    scale = (b.abs().amax((2, 4)) / FP8_MOST).clamp(min=SCALE_LEAST)
    q = (b * (1.0 / scale)[:, :, None, :, None]).view(G, -1, b.shape[3] * 128)[:, :M, :K]
    return q.contiguous().to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    op = case["op"]

    def normal(*shape, type="fp32", scale=1.0):
        return torch.empty(shape, dtype=TYPES[type], device=dev).normal_(0.0, scale, generator=g)

    def uniform(*shape):
        return torch.empty(shape, device=dev).uniform_(generator=g)

    def activations(*shape, type):
        # a few channels of a layer's activations are much larger than the others
        loud = torch.where(uniform(shape[-1]) < 0.01, 8.0, 1.0)
        return (normal(*shape) * loud).to(TYPES[type])

    def tokens_of(offsets, total, n):
        # each expert's tokens ascend
        e = torch.repeat_interleave(torch.arange(len(offsets) - 1, device=dev), torch.tensor([b - a for a, b in zip(offsets, offsets[1:])], device=dev))
        t = torch.randint(0, n, (total,), generator=g, device=dev)
        t[:len(e)] = torch.sort(e * n + t[:len(e)])[0] % n
        return t.int()

    s = dict(case)
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        x = normal(T, E, scale=1.5) + normal(E, scale=0.3)
        if case["masked"]:
            x = x.masked_fill(uniform(T, E) < case["masked"], -math.inf)
            x = x.masked_fill(uniform(T, 1) < case["masked"], -math.inf)   # tokens that go to no expert
        s["logits"] = x.to(TYPES[case["type"]])
        s["dweights"] = normal(T, k)
        for name, shape in (("experts", (T, k)), ("place", (T, k)), ("tokens", (T * k,)), ("offsets", (E + 1,))):
            s[name] = torch.empty(shape, dtype=torch.int32, device=dev)
        s["weights"] = torch.empty(T, k, device=dev)
        s["dlogits"] = torch.empty_like(s["logits"])
        # (the counts of every expert in every 16 tokens: more than the library asks for)
        s["workspace"] = torch.empty(4 * (E + 1) * (T // 16 + 2), dtype=torch.uint8, device=dev)
    elif op == "combine":
        T, k, H = case["T"], case["k"], case["H"]
        E = 64
        experts = torch.randint(0, E, (T, k), generator=g, device=dev).masked_fill(uniform(T, k) < case["masked"], -1)
        s["place"] = _by_expert(experts, E)[0]
        s["weights"] = torch.softmax(normal(T, k), 1)
        s["Y"] = normal(T * k, H, type=case["type"])
        s["dR"] = normal(T, H, type=case["type"])
        s["R"], s["dY"], s["dweights"] = torch.empty_like(s["dR"]), torch.zeros_like(s["Y"]), torch.empty(T, k, device=dev)
    elif op == "grouped":
        M, G, N, K, kind = case["M"], case["G"], case["N"], case["K"], case["type"]
        sizes = _sizes(M - case["spare"], G, int(seed))
        at = _offsets(sizes)
        s["offsets"], s["largest"] = torch.tensor(at, dtype=torch.int32, device=dev), max(sizes)
        s["rows"] = tokens_of(at, M, case["tokens"]) if case["tokens"] else None
        s["A"] = activations(case["tokens"] or M, K, type=kind)
        s["B"] = normal(*((G, N, K) if case["trans_b"] else (G, K, N)), type=kind, scale=K ** -0.5)
        out = TYPES[case["out"]]
        if case["grad"]:
            s["D"] = normal(M, N, type=kind)
            s["dA"] = torch.empty(M, K, dtype=out, device=dev)
            s["dB"] = torch.empty_like(s["B"], dtype=out)
            # (lent to the sums over many rows that few outputs have)
            s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
        else:
            s["R"] = torch.empty(M, N, dtype=out, device=dev)
    elif op == "quantize":
        G, M, K, rows = case["G"], case["M"], case["K"], case["rows"]
        s["X"] = activations(G, M, K, type=case["type"])
        s["Q"] = torch.empty(G, M, K, dtype=torch.float8_e4m3fn, device=dev)
        KB = -(-K // 128)
        # the scales of rows are kept block by block: those that a product needs at a time lie side by side
        s["scales"] = torch.empty((KB, M) if rows == 1 else (G, -(-M // 128), KB), device=dev)
    else:
        M, G, N, K = case["M"], case["G"], case["N"], case["K"]
        at = _offsets(_sizes(M, G, int(seed))) if G else [0, M]
        s["offsets"], s["largest"] = torch.tensor(at, dtype=torch.int32, device=dev), max(b - a for a, b in zip(at, at[1:]))
        s["rows"] = tokens_of(at, M, case["tokens"]) if G and case["tokens"] else None
        q, scale = _quantized(activations(1, case["tokens"] if s["rows"] is not None else M, K, type="bf16"), 1)
        s["A"], s["sa"] = q[0], scale[0].t().contiguous()
        # (expert by expert: the 32-bit values of one at a time)
        made = [_quantized(normal(1, *((N, K) if case["trans_b"] else (K, N)), type="bf16", scale=K ** -0.5), 128) for _ in range(max(G, 1))]
        s["B"], s["sb"] = torch.cat([m[0].view(torch.uint8) for m in made]).view(torch.float8_e4m3fn), torch.cat([m[1] for m in made])
        s["R"] = torch.empty(M, N, dtype=TYPES[case["out"]], device=dev)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_route(s):
    x, k, E = s["logits"].float(), s["k"], s["E"]
    top, index = torch.sort(x, dim=1, descending=True, stable=True)
    top, index = top[:, :k], index[:, :k]
    there = top > -math.inf
    experts = torch.where(there, index, -1).int()
    most = top[:, :1].clamp(min=torch.finfo(torch.float32).min)
    term = torch.exp(top - most)
    total = (term if s["norm"] else torch.exp(x - most)).sum(1, keepdim=True)
    weights = torch.where(there, term / total.clamp(min=SCALE_LEAST), 0.0)
    place, tokens, offsets = _by_expert(experts, E)
    out = [experts, weights, place, tokens, offsets]
    if s["grad"]:
        dw = torch.where(there, s["dweights"], 0.0)
        mean = (weights * dw).sum(1, keepdim=True)
        p = torch.zeros_like(x) if s["norm"] else torch.exp(x - most) / total.clamp(min=SCALE_LEAST)
        dx = -p * mean
        at = torch.where(there, index, 0)
        dx = dx.scatter_add(1, at, weights * (dw - mean) if s["norm"] else weights * dw)
        out.append(dx.to(s["logits"].dtype))
    return out


def _plain_combine(s):
    place, w = s["place"], s["weights"]
    there = place >= 0
    at = place.clamp(min=0).long()
    y = s["Y"].float()[at] * there[:, :, None]
    out = [(w[:, :, None] * y).sum(1).to(s["Y"].dtype)]
    if s["grad"]:
        d = s["dR"].float()
        # (dropped pairs land in a row past the end)
        dy = torch.zeros(s["Y"].shape[0] + 1, s["H"], dtype=s["Y"].dtype, device=place.device)
        dy[torch.where(there, place, s["Y"].shape[0]).long()] = (w[:, :, None] * d[:, None, :]).to(dy.dtype)
        dy = dy[:-1]
        out += [dy, (y * d[:, None, :]).sum(2)]
    return out


def _padded(s, M):
    """For the rows in order of expert, padded to the longest expert's: the row of each place and whether it is one;
    for each row its expert, its place there and whether it has one."""
    off, cap = s["offsets"].long(), max(s["largest"], 1)
    at = off[:-1, None] + torch.arange(cap, device=off.device)
    there = at < off[1:, None]
    i = torch.arange(M, device=off.device)
    e = (i[:, None] >= off[None, 1:]).sum(1).clamp(max=len(off) - 2)
    return at.clamp(max=M - 1), there, e, (i - off[e]).clamp(max=cap - 1), (i >= off[0]) & (i < off[-1])


def _plain_grouped(s):
    M = s["M"]
    at, there, e, slot, has = _padded(s, M)
    rows = at if s["rows"] is None else s["rows"].long()[at]
    a = s["A"].float()[rows] * there[:, :, None]
    if s["op"] == "fp8":
        K, KB = a.shape[2], s["sa"].shape[0]
        a = a * s["sa"].t()[rows].repeat_interleave(128, dim=2)[:, :, :K]
        b = s["B"].float()
        b = b * s["sb"].repeat_interleave(128, dim=1)[:, :b.shape[1]].repeat_interleave(128, dim=2)[:, :, :b.shape[2]]
    else:
        b = s["B"].float()
    out = TYPES[s["out"]]
    if not s.get("grad"):
        r = torch.bmm(a, b.transpose(1, 2) if s["trans_b"] else b)
        return [(r[e, slot] * has[:, None]).to(out)]
    d = s["D"].float()[at] * there[:, :, None]
    da = torch.bmm(d, b if s["trans_b"] else b.transpose(1, 2))
    db = torch.bmm(d.transpose(1, 2), a) if s["trans_b"] else torch.bmm(a.transpose(1, 2), d)
    return [(da[e, slot] * has[:, None]).to(out), db.to(out)]


def _plain_quantize(s):
    q, scale = _quantized(s["X"], s["rows"])
    return [q, scale[0].t().contiguous() if s["rows"] == 1 else scale]


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["op"]
    if not own:
        return {"route": _plain_route, "combine": _plain_combine, "quantize": _plain_quantize}.get(op, _plain_grouped)(s)
    import paper_2305_08872_amd as am
    if op == "route":
        am.amulet_route(s["logits"], s["experts"], s["weights"], s["place"], s["tokens"], s["offsets"], s["workspace"], norm=s["norm"])
        out = [s["experts"], s["weights"], s["place"], s["tokens"], s["offsets"]]
        if s["grad"]:
            am.amulet_route_grad(s["logits"], s["experts"], s["weights"], s["dweights"], s["dlogits"], norm=s["norm"])
            out.append(s["dlogits"])
        return out
    if op == "combine":
        am.amulet_combine(s["Y"], s["weights"], s["place"], s["R"])
        if not s["grad"]:
            return [s["R"]]
        am.amulet_combine_grad(s["Y"], s["weights"], s["place"], s["dR"], s["dY"], s["dweights"])
        return [s["R"], s["dY"], s["dweights"]]
    if op == "grouped":
        if not s["grad"]:
            am.amulet_grouped_mm(s["A"], s["B"], s["offsets"], s["R"], rows=s["rows"], trans_b=s["trans_b"])
            return [s["R"]]
        # dA = D B^T, row by row; dB = A^T D, expert by expert, in B's layout
        am.amulet_grouped_mm(s["D"], s["B"], s["offsets"], s["dA"], trans_b=not s["trans_b"])
        am.amulet_grouped_mm_wgrad(s["A"], s["D"], s["offsets"], s["dB"], s["workspace"], rows=s["rows"], trans_r=s["trans_b"])
        return [s["dA"], s["dB"]]
    if op == "quantize":
        if s["rows"] == 1:
            am.amulet_quantize_fp8(s["X"][0], s["Q"][0], s["scales"])
        else:
            am.amulet_quantize_fp8_blocks(s["X"], s["Q"], s["scales"])
        return [s["Q"], s["scales"]]
    if s["G"]:
        am.amulet_grouped_mm_fp8(s["A"], s["sa"], s["B"], s["sb"], s["offsets"], s["R"], rows=s["rows"], trans_b=s["trans_b"])
    else:
        am.amulet_mm_fp8(s["A"], s["sa"], s["B"][0], s["sb"][0], s["R"], trans_b=s["trans_b"])
    return [s["R"]]


# ------------------------------------------------------------------------------------------------ what it needs

def work(case):
    op = case["op"]
    if op == "route":
        T, E, k, e = case["T"], case["E"], case["k"], SIZE[case["type"]]
        b = T * E * e + T * k * (4 + 4 + 4 + 4) + 4 * (E + 1)
        f = T * E * 4
        if case["grad"]:
            b += T * k * 12 + T * E * e + (0 if case["norm"] else T * E * e)
            f += T * E * 4
        return {"bytes": b, "flops": f}
    if op == "combine":
        T, k, H, e = case["T"], case["k"], case["H"], SIZE[case["type"]]
        live = T * k * (1 - case["masked"])
        b, f = live * H * e + T * H * e + 8 * T * k, 2 * live * H
        if case["grad"]:
            b, f = b + 2 * live * H * e + T * H * e + 12 * T * k, f + 3 * live * H
        return {"bytes": b, "flops": f}
    if op == "quantize":
        n = case["G"] * case["M"] * case["K"]
        return {"bytes": n * (SIZE[case["type"]] + 1) + 4 * n // (128 * case["rows"]), "flops": 3 * n}
    M, G, N, K = case["M"], case["G"], case["N"], case["K"]
    live = M - case.get("spare", 0)
    # experts that get a row at all
    busy = sum(1 - (1 - p) ** live for p in _shares(G)) if G else 1
    gathered = case["tokens"] if G else 0
    # rows of A that some pair reads
    read = gathered * (1 - (1 - 1 / gathered) ** live) if gathered else live
    extra = 4 * M * (1 if gathered else 0) + 4 * (G + 1)
    if op == "fp8":
        return {"bytes": read * K * (1 + 4 / 128) + busy * N * K * (1 + 4 / 128 ** 2) + M * N * SIZE[case["out"]] + extra, "flops": 2 * live * N * K}
    e, o = SIZE[case["type"]], SIZE[case["out"]]
    if case["grad"]:
        return {"bytes": e * (read * K + 2 * live * N + busy * N * K) + o * (M * K + G * N * K) + extra, "flops": 4 * live * N * K}
    return {"bytes": e * (read * K + busy * N * K) + o * M * N + extra, "flops": 2 * live * N * K}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        x = s["logits"].double()
        # every expert's rank in its row: how many have a higher logit, or the same and a lower index
        low = torch.arange(x.shape[1], device=x.device)
        rank = torch.stack([((x > c[:, None]) | ((x == c[:, None]) & (low < e))).sum(1) for e, c in enumerate(x.unbind(1))], 1)
        chosen = (rank < case["k"]) & (x > -math.inf)
        base = chosen if case["norm"] else x > -math.inf
        shift = torch.where(x > -math.inf, x, 0.0).amax(1, keepdim=True)
        term = torch.where(base, torch.exp(x - shift), 0.0)
        p = term / term.sum(1, keepdim=True).clamp(min=1e-300)
        w = torch.zeros(case["T"], case["k"] + 1, dtype=torch.float64, device=x.device)
        slot = torch.where(chosen, rank, case["k"])
        w.scatter_(1, slot, torch.where(chosen, p, 0.0))
        out = [None, w[:, :-1], None, None, None]
        if case["grad"]:
            up = torch.cat([s["dweights"].double(), torch.zeros(case["T"], 1, dtype=torch.float64, device=x.device)], 1).gather(1, slot)
            out.append(p * (up - (p * up).sum(1, keepdim=True)))
        return out
    if op == "combine":
        y, w, d, at = s["Y"].double(), s["weights"].double(), s["dR"].double(), s["place"].long()
        r, dy, dw = torch.zeros_like(d), torch.zeros_like(y), torch.zeros_like(w)
        for j in range(case["k"]):
            t = (at[:, j] >= 0).nonzero()[:, 0]
            rows = at[t, j]
            r[t] += w[t, j, None] * y[rows]
            dy[rows] = w[t, j, None] * d[t]
            dw[t, j] = (y[rows] * d[t]).sum(1)
        return [r, dy, dw] if case["grad"] else [r]
    if op == "quantize":
        x = s["X"].double()
        G, M, K = x.shape
        rows = case["rows"]
        MB, KB = -(-M // rows), -(-K // 128)
        top = torch.zeros(G, MB * rows, KB * 128, dtype=torch.float64, device=x.device)
        top[:, :M, :K] = x.abs()
        scale = (top.view(G, MB, rows, KB, 128).amax(4).amax(2) / FP8_MOST).clamp(min=SCALE_LEAST)
        v = x / scale.repeat_interleave(rows, 1)[:, :M].repeat_interleave(128, 2)[:, :, :K]
        # to the nearest multiple of the step of v's octave, 2^-9 at least
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        return [torch.round(v / step) * step, scale[0].t() if rows == 1 else scale]
    at, a = s["offsets"].tolist(), s["A"]
    M = case["M"]

    def left(i, j):
        rows = slice(i, j) if s["rows"] is None else s["rows"][i:j].long()
        v = a[rows].double()
        return v if op == "grouped" else v * s["sa"].t()[rows].double().repeat_interleave(128, 1)[:, :v.shape[1]]

    def right(g):
        v = s["B"][g].double()
        if op == "fp8":
            v = v * s["sb"][g].double().repeat_interleave(128, 0)[:v.shape[0]].repeat_interleave(128, 1)[:, :v.shape[1]]
        return v.t() if case["trans_b"] else v

    if not case.get("grad"):
        r = torch.zeros(M, case["N"], dtype=torch.float64, device=a.device)
        for g, (i, j) in enumerate(zip(at, at[1:])):
            if j > i:
                r[i:j] = left(i, j) @ right(g)
        return [r]
    da = torch.zeros(M, case["K"], dtype=torch.float64, device=a.device)
    db = torch.zeros(s["B"].shape, dtype=torch.float64, device=a.device)
    for g, (i, j) in enumerate(zip(at, at[1:])):
        if j > i:
            d = s["D"][i:j].double()
            da[i:j] = d @ right(g).t()
            db[g] = d.t() @ left(i, j) if case["trans_b"] else left(i, j).t() @ d
    return [da, db]
