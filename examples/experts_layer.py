"""A mixture-of-experts layer on the library's operators: forward, backward and an 8-bit forward pass.

    y[t] = sum over the k experts e of token t:  weight[t, e] * W2[e]^T silu(W1[e]^T x[t])

Run on the GPU: trains the layer for a few steps to reproduce a fixed one and prints the loss, then
compares the 8-bit forward pass with the 16-bit one.

    python examples/experts_layer.py [tokens] [width] [hidden width] [experts] [experts of a token]
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2305_08872_amd as am  # noqa: E402


def silu(h):
    h = h.float()
    return h * torch.sigmoid(h)


def silu_slope(h):
    s = torch.sigmoid(h.float())
    return s * (1 + h.float() * (1 - s))


class Layer:
    """Weights of a layer and, between forward and backward, what the backward pass reads again."""

    def __init__(self, width, hidden, experts, k, seed=0, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, scale):
            return torch.empty(shape, device="cuda").normal_(0, scale, generator=g)

        self.k, self.experts = k, experts
        self.router = normal(width, experts, scale=width ** -0.5)                  # fp32
        self.w1 = normal(experts, width, hidden, scale=width ** -0.5).to(dtype)    # [expert][in][out]
        self.w2 = normal(experts, hidden, width, scale=hidden ** -0.5).to(dtype)

    def route(self, x):
        T, E, k = x.shape[0], self.experts, self.k
        i32 = dict(dtype=torch.int32, device=x.device)
        self.logits = x.float() @ self.router
        self.chosen, self.place = torch.empty(T, k, **i32), torch.empty(T, k, **i32)
        self.tokens, self.offsets = torch.empty(T * k, **i32), torch.empty(E + 1, **i32)
        self.weights = torch.empty(T, k, device=x.device)
        space = torch.empty(am.amulet_route_workspace_bytes(T, E), dtype=torch.uint8, device=x.device)
        am.amulet_route(self.logits, self.chosen, self.weights, self.place, self.tokens, self.offsets, space)

    def forward(self, x):
        self.x = x
        self.route(x)
        rows, width, hidden = len(self.tokens), x.shape[1], self.w1.shape[2]
        self.h = torch.empty(rows, hidden, dtype=x.dtype, device=x.device)
        am.amulet_grouped_mm(x, self.w1, self.offsets, self.h, rows=self.tokens)   # each expert's tokens, gathered
        self.a = silu(self.h).to(x.dtype)
        self.y = torch.empty(rows, width, dtype=x.dtype, device=x.device)
        am.amulet_grouped_mm(self.a, self.w2, self.offsets, self.y)
        out = torch.empty_like(x)
        am.amulet_combine(self.y, self.weights, self.place, out)
        return out

    def backward(self, dout):
        """Gradients of x, router, w1, w2 for the last forward pass."""
        x, dev = self.x, dout.device
        dy, dweights = torch.empty_like(self.y), torch.empty_like(self.weights)
        am.amulet_combine_grad(self.y, self.weights, self.place, dout, dy, dweights)
        da = torch.empty_like(self.a)
        am.amulet_grouped_mm(dy, self.w2, self.offsets, da, trans_b=True)          # W2 read the other way
        dh = (da.float() * silu_slope(self.h)).to(x.dtype)
        dxr = torch.empty_like(self.y)
        am.amulet_grouped_mm(dh, self.w1, self.offsets, dxr, trans_b=True)
        dx = torch.empty_like(x)
        am.amulet_combine(dxr, None, self.place, dx)                               # a token's rows added up
        (E, K, N), M = self.w1.shape, len(self.tokens)
        space = torch.empty(max(am.amulet_grouped_mm_wgrad_workspace_bytes(M, N, K, E), am.amulet_grouped_mm_wgrad_workspace_bytes(M, K, N, E)),
                            dtype=torch.uint8, device=dev)
        dw1, dw2 = torch.empty(self.w1.shape, device=dev), torch.empty(self.w2.shape, device=dev)   # fp32
        am.amulet_grouped_mm_wgrad(x, dh, self.offsets, dw1, space, rows=self.tokens)
        am.amulet_grouped_mm_wgrad(self.a, dy, self.offsets, dw2, space)
        dlogits = torch.empty_like(self.logits)
        am.amulet_route_grad(None, self.chosen, self.weights, dweights, dlogits)
        dx = (dx.float() + dlogits @ self.router.t()).to(x.dtype)
        return dx, x.float().t() @ dlogits, dw1, dw2

    # -------------------------------------------------------------------------------- 8 bits, for serving

    def quantize(self):
        def blocks(w):
            q = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=w.device)
            s = torch.empty(w.shape[0], -(-w.shape[1] // 128), -(-w.shape[2] // 128), device=w.device)
            am.amulet_quantize_fp8_blocks(w, q, s)
            return q, s
        self.q1, self.q2 = blocks(self.w1), blocks(self.w2)

    def forward_8bit(self, x):
        def rows(v):
            q = torch.empty(v.shape, dtype=torch.float8_e4m3fn, device=v.device)
            s = torch.empty(-(-v.shape[1] // 128), v.shape[0], device=v.device)
            am.amulet_quantize_fp8(v, q, s)
            return q, s
        self.route(x)
        n = len(self.tokens)
        h = torch.empty(n, self.w1.shape[2], dtype=x.dtype, device=x.device)
        am.amulet_grouped_mm_fp8(*rows(x), *self.q1, self.offsets, h, rows=self.tokens)
        y = torch.empty(n, x.shape[1], dtype=x.dtype, device=x.device)
        am.amulet_grouped_mm_fp8(*rows(silu(h).to(x.dtype)), *self.q2, self.offsets, y)
        out = torch.empty_like(x)
        am.amulet_combine(y, self.weights, self.place, out)
        return out


def main(tokens=2048, width=512, hidden=1024, experts=16, k=4, steps=20, rate=0.2):
    goal, layer = Layer(width, hidden, experts, k, seed=1), Layer(width, hidden, experts, k, seed=2)
    layer.router.copy_(goal.router)
    w1, w2 = layer.w1.float(), layer.w2.float()      # (masters of the 16-bit weights)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    losses = []
    for step in range(steps):
        x = torch.empty(tokens, width, device="cuda").normal_(generator=g).bfloat16()
        want = goal.forward(x)
        off = layer.forward(x).float() - want.float()
        losses.append(float(off.square().mean()))
        _, _, dw1, dw2 = layer.backward((off * (2 / tokens)).bfloat16())
        w1 -= rate * dw1
        w2 -= rate * dw2
        layer.w1, layer.w2 = w1.bfloat16(), w2.bfloat16()
        print("step %2d  loss %.4f" % (step, losses[-1]), flush=True)
    layer.quantize()
    y16, y8 = layer.forward(x).float(), layer.forward_8bit(x).float()
    off = float((y8 - y16).norm() / y16.norm())
    print("8-bit forward pass: %.3f off the 16-bit one (2-norm)" % off)
    return losses, off


if __name__ == "__main__":
    main(*[int(v) for v in sys.argv[1:6]])
