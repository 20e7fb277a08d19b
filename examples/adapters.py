"""Low-rank adapters of several tasks beside one shared projection, on the library's operators: trained together, then served.

    y[i] = W x[i] + scale * B[a] A[a] x[i]        a: the adapter of row i's sequence, or none

Run on the GPU: trains the adapters of a few tasks for some steps, each to turn the shared projection into one of its own, with the
gradients clipped to a largest norm, and prints the losses; then decodes a batch of single tokens, each with the adapter it asks for.

    python examples/adapters.py [rows] [width] [outputs] [rank] [tasks]
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2305_08872_amd as am  # noqa: E402


class Rows:
    """Which rows have which adapter: `lengths` of neighbouring rows, `adapters` of each (-1: none)."""

    def __init__(self, lengths, adapters, device="cuda"):
        at = [0]
        for n in lengths:
            at.append(at[-1] + n)
        self.offsets = torch.tensor(at, dtype=torch.int32, device=device)
        self.adapters = torch.tensor(adapters, dtype=torch.int32, device=device)


class Apply(torch.autograd.Function):
    """The projection with its adapters; gradients of x, A and B (W stays as it is)."""

    @staticmethod
    def forward(ctx, x, w, a, b, scales, rows):
        t = torch.empty(x.shape[0], a.shape[1], device=x.device)
        y = torch.empty(x.shape[0], w.shape[0], dtype=x.dtype, device=x.device)
        am.amulet_adapters_mm(x, w, a, b, rows.offsets, t, y, adapters=rows.adapters, scales=scales, trans_w=True, trans_a=True, trans_b=True)
        ctx.save_for_backward(x, w, a, b, scales, t)
        ctx.rows = rows
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, a, b, scales, t = ctx.saved_tensors
        rows, dy = ctx.rows, dy.contiguous()
        u, dx = torch.empty_like(t), torch.empty_like(x)
        # the same product with W read the other way, A and B exchanged and read the other way
        am.amulet_adapters_mm(dy, w, b, a, rows.offsets, u, dx, adapters=rows.adapters, scales=scales)
        da, db = torch.empty_like(a), torch.empty_like(b)
        need = max(am.amulet_adapters_wgrad_workspace_bytes(len(x), n, a.shape[1], len(a)) for n in (x.shape[1], w.shape[0]))
        space = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        am.amulet_adapters_wgrad(x, u, rows.offsets, da, space, adapters=rows.adapters, trans_r=True)
        am.amulet_adapters_wgrad(dy, t, rows.offsets, db, space, adapters=rows.adapters)
        return dx, None, da, db, None, None


def clip(grads, max_norm):
    """Scales the gradients down to max_norm together; their norm before."""
    norm = torch.empty(1, device=grads[0].device)
    space = torch.empty(am.amulet_grad_norm_workspace_bytes(len(grads)), dtype=torch.uint8, device=norm.device)
    am.amulet_grad_norm_clip(grads, max_norm, norm, space)
    return norm


def main(rows=2048, width=512, outputs=640, rank=16, tasks=4, steps=8):
    g = torch.Generator(device="cuda")
    g.manual_seed(0)

    def normal(*shape, scale=1.0):
        return torch.empty(shape, device="cuda").normal_(0, scale, generator=g).bfloat16()

    w = normal(outputs, width, scale=width ** -0.5)
    targets = [normal(outputs, rank, scale=0.5) @ normal(rank, width, scale=width ** -0.5) for _ in range(tasks)]
    a = normal(tasks, rank, width, scale=width ** -0.5).requires_grad_()
    b = torch.zeros(tasks, outputs, rank, dtype=torch.bfloat16, device="cuda").requires_grad_()
    scales = torch.full((tasks,), 2.0, device="cuda")
    # two sequences of each task, and some rows without an adapter
    lengths = [max(1, rows // (2 * tasks + 1))] * (2 * tasks) + [1]
    which = Rows(lengths, [i % tasks for i in range(2 * tasks)] + [-1])
    x = normal(sum(lengths), width)
    parts = x.split(lengths)
    wanted = torch.cat([p @ (w + targets[i % tasks]).t() if i < 2 * tasks else p @ w.t() for i, p in enumerate(parts)])
    losses = []
    for _ in range(steps):
        y = Apply.apply(x, w, a, b, scales, which)
        loss = (y.float() - wanted.float()).square().mean()
        da, db = torch.autograd.grad(loss, (a, b))
        norm = clip([da, db], 1.0)
        with torch.no_grad():
            a -= 0.5 * da
            b -= 0.5 * db
        losses.append(float(loss.detach()))
        print("loss %.4f  gradients' norm %.3f" % (losses[-1], float(norm)))
    # a batch of single tokens
    batch = Rows([1] * 8, [i % (tasks + 1) - 1 for i in range(8)])
    with torch.no_grad():
        y = Apply.apply(x[:8], w, a, b, scales, batch)
    print("decoded %d tokens, %s" % (len(y), am.amulet_recent_kernel()))
    return losses, y


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:]))
