"""The operators that train and serve low-rank adapters beside a shared projection, as cases that can be timed.

  adapters    R[i] = X[i] W + T[i] B[a(i)], T[i] = scale[a(i)] X[i] A[a(i)]: a batch of requests, each with the adapter
              it asked for or none, through one projection
  gradients   of the same: of the rows (and U, what T is on the way back), of every adapter's two matrices
  norm, clip  the norm of all gradients of a step together, and the gradients scaled down to a largest norm

  own               whether run() calls the library or computes the plain form
  listed()          the cases
  draw(rng)         one more case of the same ranges
  prepare(case, s)  what a program has in hand before the call, from seed s
  run(state)        one pass; returns the outputs
  work(case)        bytes and operations that no implementation can do without
  exact(case, s)    run()'s outputs from the definition in 64 bits

M rows lie in S segments of neighbouring rows (a request's tokens), the last `spare` in none.  Segment s has adapter
adapters[s] of G, or none (-1); with `direct` segment s has adapter s.  `trans`: the matrices are stored as N x K, r x K and
N x r, else as K x N, K x r and r x N.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # eight sequences decode a token each, each with an adapter of its own: latency
        dict(name="adapters_decode", op="adapters", M=8, N=4096, K=4096, r=16, G=8, S=8, spare=0, none=0.0, direct=True, type="bf16", out="bf16", trans=True),
        # a server's step: 192 sequences, 64 adapters, a quarter without one, rows that pad the batch
        dict(name="adapters_serve", op="adapters", M=208, N=4096, K=4096, r=32, G=64, S=192, spare=16, none=0.25, direct=False, type="bf16", out="bf16", trans=True),
        # the prompts of 24 requests, some with the same adapter
        dict(name="adapters_prompt", op="adapters", M=8192, N=8192, K=4096, r=64, G=16, S=24, spare=0, none=0.1, direct=False, type="bf16", out="bf16", trans=True),
        # sizes as they fall, fp16, results kept in 32 bits, the matrices stored the other way
        dict(name="adapters_odd", op="adapters", M=1501, N=1367, K=1003, r=20, G=5, S=13, spare=11, none=0.2, direct=False, type="fp16", out="fp32", trans=False),
        # the backward pass of a training batch over four adapters at once
        dict(name="gradients_train", op="gradients", M=16384, N=4096, K=4096, r=16, G=4, S=4, spare=0, none=0.0, direct=True, type="bf16", out="bf16", trans=True),
        # many short sequences, adapters that several of them share, gradients kept in 32 bits
        dict(name="gradients_shared", op="gradients", M=4096, N=2048, K=4096, r=64, G=8, S=32, spare=0, none=0.1, direct=False, type="bf16", out="fp32", trans=True),
        # sizes as they fall, the matrices stored the other way
        dict(name="gradients_odd", op="gradients", M=777, N=1001, K=643, r=9, G=3, S=7, spare=5, none=0.2, direct=False, type="fp16", out="fp16", trans=False),
        # the adapters' own gradients: 128 tensors of a few rows
        dict(name="clip_adapters", op="clip", n=128, total=2 ** 23, types="fp32", odd=False, clip=True),
        # the gradients of half a billion weights, most in a few large matrices
        dict(name="clip_model", op="clip", n=290, total=2 ** 29, types="bf16", odd=False, clip=True),
        # gradients of several types and any length, already small enough: the same values
        dict(name="clip_mixed", op="clip", n=77, total=10 ** 7, types="mixed", odd=True, clip=False),
        # the norm alone, which a step over several cards joins before it clips
        dict(name="norm_model", op="norm", n=150, total=2 ** 28, types="bf16", odd=False, clip=False),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """The width of a layer: mostly whole 64s or 8s, one in six as it falls."""
    n, kind = _log(rng, low, high), rng.random()
    return max(64, n // 64 * 64) if kind < 0.6 else max(8, n // 8 * 8) if kind < 0.84 else n


def draw(rng):
    """One to 16384 rows, 1 to 128 adapters of rank 1 to 128, widths of 64 to 8192; 1 to 400 gradients, 1000 to 2^28 values."""
    op = rng.choice(["adapters", "adapters", "adapters", "gradients", "gradients", "clip", "clip", "norm"])
    if op in ("clip", "norm"):
        total = _log(rng, 1000, 2 ** 28)
        return dict(op=op, n=min(_log(rng, 1, 400), total), total=total, types=rng.choice(["bf16", "fp16", "fp32", "mixed"]), odd=rng.random() < 0.5,
                    clip=op == "clip" and rng.random() < 0.7)
    while True:
        M, N, K, G = _log(rng, 1, 16384), _width(rng, 64, 8192), _width(rng, 64, 8192), _log(rng, 1, 128)
        r = rng.choice([4, 8, 16, 16, 32, 64]) if rng.random() < 0.7 else rng.randint(1, 128)
        if M * N * K <= 2 ** (38 if op == "adapters" else 37) and G * (N + K) * r <= 2 ** 27:
            break
    direct = rng.random() < 0.3
    S = G if direct else M if M <= 256 and rng.random() < 0.5 else _log(rng, 1, max(1, min(M, 256)))
    kind = rng.choice(["bf16", "bf16", "fp16"])
    spare = rng.choice([0, 0, M // 20])
    if S == M and not direct:
        S -= spare   # (a token to each segment)
    return dict(op=op, M=M, N=N, K=K, r=r, G=G, S=S, spare=spare, none=0.0 if direct else rng.choice([0.0, 0.1, 0.5]), direct=direct,
                type=kind, out=rng.choice([kind, kind, "fp32"]), trans=rng.random() < 0.6)


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(case, seed):
    """Rows of every segment: one each where there are as many as rows, else uneven, as requests are."""
    S, M = case["S"], case["M"] - case["spare"]
    if S == M:
        return [1] * S
    rng = random.Random(int(seed) * 1000003 + M * 31 + S)
    share = [0.3 + rng.expovariate(1.0) for _ in range(S)]
    n = [int(M * x / sum(share)) for x in share]
    for i in range(M - sum(n)):
        n[i % S] += 1
    return n


def _tensors(case):
    """(values, type) of every gradient: matrices of unequal size, and small vectors among them."""
    n, total = case["n"], case["total"]
    rng = random.Random(total * 31 + n)
    share = [math.exp(rng.gauss(0.0, 1.5)) for _ in range(n)]
    most = sum(share)
    counts = [max(1, int(total * x / most)) for x in share]
    if not case["odd"]:
        counts = [max(64, c // 64 * 64) for c in counts]
    return [(c, rng.choice(_kinds(case))) for c in counts]


def _kinds(case):
    return ["bf16", "fp16", "fp32"] if case["types"] == "mixed" else [case["types"]]


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    s = dict(case)

    def normal(*shape, type="fp32", scale=1.0):
        return torch.empty(shape, dtype=TYPES[type], device=dev).normal_(0.0, scale, generator=g)

    def activations(rows, cols, type):
        # a few channels of a layer's activations are much larger than the others
        loud = torch.where(torch.empty(cols, device=dev).uniform_(generator=g) < 0.01, 8.0, 1.0)
        return (normal(rows, cols) * loud).to(TYPES[type])

    if case["op"] in ("clip", "norm"):
        tensors = _tensors(case)
        # (unequal from layer to layer)
        s["grads"] = [normal(c, type=t, scale=0.01 * (1 + i % 7)) for i, (c, t) in enumerate(tensors)]
        # (the clipped ones lie one behind the other, in a buffer for each type)
        s["buffers"] = [torch.empty(sum(c for c, t in tensors if t == k), dtype=TYPES[k], device=dev) for k in _kinds(case)] if case["op"] == "clip" else []
        at = [0] * len(s["buffers"])
        s["outs"] = []
        for c, t in tensors if case["op"] == "clip" else []:
            k = _kinds(case).index(t)
            s["outs"].append(s["buffers"][k][at[k]:at[k] + c])
            at[k] += c
        expected = math.sqrt(sum(c * (0.01 * (1 + i % 7)) ** 2 for i, (c, _) in enumerate(tensors)))
        s["max_norm"] = 0.3 * expected if case["clip"] else 4.0 * expected
        s["norm"] = torch.empty(1, device=dev)
        # (a sum to every workgroup of a launch: more than the library asks for)
        s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
        return s
    M, N, K, r, G, S, kind = (case[x] for x in ("M", "N", "K", "r", "G", "S", "type"))
    at = [0]
    for n in _lengths(case, seed):
        at.append(at[-1] + n)
    s["largest"] = max(b - a for a, b in zip(at, at[1:]))
    s["offsets"] = torch.tensor(at, dtype=torch.int32, device=dev)
    if case["direct"]:
        s["adapters"] = None
    else:
        chosen = torch.randint(0, G, (S,), generator=g, device=dev)
        s["adapters"] = chosen.masked_fill(torch.empty(S, device=dev).uniform_(generator=g) < case["none"], -1).int()
    s["scales"] = torch.empty(G, device=dev).uniform_(0.25, 4.0, generator=g)
    s["X"] = activations(M, K, kind)
    s["W"] = normal(*((N, K) if case["trans"] else (K, N)), type=kind, scale=K ** -0.5)
    s["A"] = normal(*((G, r, K) if case["trans"] else (G, K, r)), type=kind, scale=K ** -0.5)
    s["B"] = normal(*((G, N, r) if case["trans"] else (G, r, N)), type=kind, scale=0.3 * r ** -0.5)
    out = TYPES[case["out"]]
    if case["op"] == "adapters":
        s["T"] = torch.empty(M, r, device=dev)
        s["R"] = torch.empty(M, N, dtype=out, device=dev)
        return s
    s["dR"] = normal(M, N, type=kind)
    s["T"] = _down(s, s["X"], s["A"], case["trans"])   # (what the forward pass left)
    s["U"] = torch.empty(M, r, device=dev)
    s["dX"] = torch.empty(M, K, dtype=out, device=dev)
    s["dA"], s["dB"] = torch.empty_like(s["A"], dtype=out), torch.empty_like(s["B"], dtype=out)
    # (lent to the sums over many rows that few outputs have)
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _segments(s):
    """The rows of every segment, padded to the longest one's, and whether there is one with an adapter; the adapter of
    each; for each row its segment, its place there and whether it has an adapter."""
    off, M, cap = s["offsets"].long(), s["M"], max(s["largest"], 1)
    S = off.shape[0] - 1
    adapter = torch.arange(S, device=off.device) if s["adapters"] is None else s["adapters"].long()
    at = off[:-1, None] + torch.arange(cap, device=off.device)
    there = (at < off[1:, None]) & (adapter >= 0)[:, None]
    i = torch.arange(M, device=off.device)
    seg = (i[:, None] >= off[None, 1:]).sum(1).clamp(max=S - 1)
    has = (i < off[-1]) & (adapter[seg] >= 0)
    return at.clamp(max=M - 1), there, adapter.clamp(min=0), seg, (i - off[seg]).clamp(max=cap - 1), has


def _by_segment(s, rows, matrices):
    """rows[i] times the matrix (in 32 bits) of its row's adapter, zeros without one."""
    at, there, adapter, seg, slot, has = _segments(s)
    r = torch.bmm(rows.float()[at] * there[:, :, None], matrices[adapter])
    return r[seg, slot] * has[:, None]


def _down(s, x, a, transposed):
    """Rows times their adapters' first matrices and scales, 32 bits."""
    m = a.float() * s["scales"][:, None, None]
    return _by_segment(s, x, m.transpose(1, 2) if transposed else m)


def _plain_adapters(s):
    w, b = s["W"].float(), s["B"].float()
    if s["trans"]:
        w, b = w.t(), b.transpose(1, 2)
    t = _down(s, s["X"], s["A"], s["trans"])
    return [(s["X"].float() @ w + _by_segment(s, t, b)).to(TYPES[s["out"]]), t]


def _outer(s, x, t):
    """For every adapter the sum over its rows of x[i]^T t[i], G x columns of x x columns of t, 32 bits."""
    at, there, adapter, _, _, _ = _segments(s)
    each = torch.bmm((x.float()[at] * there[:, :, None]).transpose(1, 2), t[at] * there[:, :, None])
    out = torch.zeros(s["G"], x.shape[1], t.shape[1], device=x.device)
    return out.index_add(0, adapter, each)


def _plain_gradients(s):
    w, a = s["W"].float(), s["A"].float()
    if not s["trans"]:
        w, a = w.t(), a.transpose(1, 2)   # N x K, G x r x K
    u = _down(s, s["dR"], s["B"], not s["trans"])
    dx = s["dR"].float() @ w + _by_segment(s, u, a)
    da, db = _outer(s, s["X"], u), _outer(s, s["dR"], s["T"])   # G x K x r, G x N x r
    da, db = (da.transpose(1, 2), db) if s["trans"] else (da, db.transpose(1, 2))
    out = TYPES[s["out"]]
    return [dx.to(out), u, da.to(out), db.to(out)]


def _plain_norm(s):
    # (in 64 bits: a long sum)
    return torch.stack([(x.double() ** 2).sum() for x in s["grads"]]).sum().sqrt()


def _joined(s, clipped):
    """A buffer for each type, as prepare() lays them out."""
    empty = [clipped[0][:0]]   # (a type that no tensor has)
    of = [[x for x, g in zip(clipped, s["grads"]) if g.dtype == TYPES[k]] for k in _kinds(s)]
    return [torch.cat(x or empty) for x in of]


def _plain_clip(s):
    norm = _plain_norm(s).float()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return [norm.reshape(1)] + _joined(s, [(x.float() * factor).to(x.dtype) for x in s["grads"]])


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    op = s["op"]
    if not own:
        if op == "norm":
            return [_plain_norm(s).float().reshape(1)]
        return {"adapters": _plain_adapters, "gradients": _plain_gradients, "clip": _plain_clip}[op](s)
    import paper_2305_08872_amd as am
    if op == "norm":
        am.amulet_grad_norm(s["grads"], s["norm"], s["workspace"])
        return [s["norm"]]
    if op == "clip":
        am.amulet_grad_norm_clip(s["grads"], s["max_norm"], s["norm"], s["workspace"], outs=s["outs"])
        return [s["norm"]] + s["buffers"]
    t = s["trans"]
    if op == "adapters":
        am.amulet_adapters_mm(s["X"], s["W"], s["A"], s["B"], s["offsets"], s["T"], s["R"], adapters=s["adapters"], scales=s["scales"],
                              trans_w=t, trans_a=t, trans_b=t)
        return [s["R"], s["T"]]
    # dX = dR W^T + U A^T, U = scale dR B^T: the same product with the matrices read the other way and exchanged
    am.amulet_adapters_mm(s["dR"], s["W"], s["B"], s["A"], s["offsets"], s["U"], s["dX"], adapters=s["adapters"], scales=s["scales"],
                          trans_w=not t, trans_a=not t, trans_b=not t)
    # dA = X^T U and dB^T = dR^T T, adapter by adapter, in the layout of A and B
    am.amulet_adapters_wgrad(s["X"], s["U"], s["offsets"], s["dA"], s["workspace"], adapters=s["adapters"], trans_r=t)
    am.amulet_adapters_wgrad(s["dR"], s["T"], s["offsets"], s["dB"], s["workspace"], adapters=s["adapters"], trans_r=not t)
    return [s["dX"], s["U"], s["dA"], s["dB"]]


# ------------------------------------------------------------------------------------------------ what it needs

def work(case):
    if case["op"] in ("clip", "norm"):
        tensors = _tensors(case)
        b = sum(c * SIZE[t] for c, t in tensors)
        n = sum(c for c, _ in tensors)
        return {"bytes": 2 * b + 4, "flops": 3 * n} if case["op"] == "clip" else {"bytes": b + 4, "flops": 2 * n}
    M, N, K, r, G, S = (case[x] for x in ("M", "N", "K", "r", "G", "S"))
    e, o = SIZE[case["type"]], SIZE[case["out"]]
    live = (M - case["spare"]) * (1 - case["none"])
    # adapters that some segment has
    busy = min(live, G if case["direct"] else G * (1 - (1 - 1 / G) ** (S * (1 - case["none"]))))
    index = 4 * (S + 1) + (0 if case["direct"] else 4 * S) + 4 * G
    if case["op"] == "adapters":
        return {"bytes": e * (M * K + N * K + busy * r * (N + K)) + o * M * N + 4 * M * r + index, "flops": 2 * M * N * K + 2 * live * r * (N + K)}
    # dR and W, X and T, the adapters' matrices; dX, U and their gradients
    return {"bytes": e * (M * N + N * K + M * K + busy * r * (N + K)) + o * (M * K + G * r * (N + K)) + 8 * M * r + index,
            "flops": 2 * M * N * K + 4 * live * r * (N + K)}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("clip", "norm"):
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for x in s["grads"]:
            for part in x.split(1 << 26):
                total += part.double().square().sum()
        norm = total.sqrt()
        if case["op"] == "norm":
            return [norm.reshape(1)]
        factor = float(torch.clamp(s["max_norm"] / norm, max=1.0))
        return [norm.reshape(1)] + _joined(s, [x.double() * factor for x in s["grads"]])
    trans, M = case["trans"], case["M"]
    at = s["offsets"].tolist()
    which = list(range(case["S"])) if s["adapters"] is None else s["adapters"].tolist()
    scales = s["scales"].double()
    # K x N, G x K x r, G x r x N
    w, a, b = (s[x].double().transpose(-1, -2) if trans else s[x].double() for x in ("W", "A", "B"))
    spans = [(slice(i, j), g) for i, j, g in zip(at, at[1:], which) if j > i and g >= 0]
    if case["op"] == "adapters":
        x = s["X"].double()
        r, t = x @ w, torch.zeros(M, case["r"], dtype=torch.float64, device=x.device)
        for rows, g in spans:
            t[rows] = (x[rows] @ a[g]) * scales[g]
            r[rows] += t[rows] @ b[g]
        return [r, t]
    d, x, t = s["dR"].double(), s["X"].double(), s["T"].double()
    dx, u = d @ w.t(), torch.zeros(M, case["r"], dtype=torch.float64, device=d.device)
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for rows, g in spans:
        u[rows] = (d[rows] @ b[g].t()) * scales[g]
        dx[rows] += u[rows] @ a[g].t()
        da[g] += x[rows].t() @ u[rows]
        db[g] += t[rows].t() @ d[rows]
    return [dx, u, da.transpose(1, 2), db.transpose(1, 2)] if trans else [dx, u, da, db]
