"""Training steps of several MoE layers that share one stash, and of experts of one's own between dispatch and combine.

    python examples/packed_stash_training.py [--tokens 1000] [--layers 3]

Every routed layer keeps G and U of its rows in 8 bits (at most 0.35 of the stash) and the backward pass unpacks them into the stash that all layers use.  The last layer's experts are torch's:
tokens go to the rows of their experts and back with moe_dispatch_* and moe_combine_*, whose gradients torch's autograd calls.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
import paper_2604_19241_amd as moe  # noqa: E402


class Dispatch(torch.autograd.Function):
    """x [T,d] -> rows [T k,d] in the order of the routing; rows behind the last one are zeros."""

    @staticmethod
    def forward(ctx, x, row_of):
        ctx.shape = moe.make_dispatch_shape(*row_of.shape, x.shape[1])
        ctx.save_for_backward(row_of)
        return moe.moe_dispatch_forward(ctx.shape, x, row_of, out=x.new_zeros((row_of.numel(), x.shape[1])))

    @staticmethod
    def backward(ctx, dxs):
        return moe.moe_dispatch_backward(ctx.shape, dxs.contiguous(), ctx.saved_tensors[0]), None


class Combine(torch.autograd.Function):
    """Rows and weights [T,k] -> y[t] = sum_j weights[t,j] rows[row_of[t,j]]."""

    @staticmethod
    def forward(ctx, rows, weights, row_of):
        ctx.shape = moe.make_dispatch_shape(*row_of.shape, rows.shape[1])
        ctx.save_for_backward(rows, weights, row_of)
        return moe.moe_combine_forward(ctx.shape, rows, row_of, weights)

    @staticmethod
    def backward(ctx, dy):
        rows, weights, row_of = ctx.saved_tensors
        got = moe.moe_combine_backward(ctx.shape, dy.contiguous(), rows, row_of, weights, out={"do": torch.zeros_like(rows)})
        return got["do"], got["dw"], None


def own_experts(x, routing, w, weights=None):
    """One projection [d,d] an expert, tanh: y[t] = sum_j weights[t,j] tanh(x[t] w[e])."""
    rows = Dispatch.apply(x, routing.inv_perm)
    at = routing.offsets.tolist()
    out = torch.cat([torch.tanh(rows[a:b] @ w[e]) for e, (a, b) in enumerate(zip(at, at[1:]))] + [rows[at[-1]:]])
    return Combine.apply(out, routing.topk_w if weights is None else weights, routing.inv_perm)


class RoutedLayer:
    """x + experts(x) with the fused layer; what its backward pass needs is kept in 8 bits."""

    def __init__(self, T, d, E, k, I, stash, g):
        self.shape, self.stash = moe.make_shape(T, d, E, k, I), stash
        normal = lambda *s: (torch.randn(s, generator=g, device="cuda") * s[-2] ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.w, self.router = [normal(E, d, I), normal(E, d, I), normal(E, I, d)], normal(d, E)

    def forward(self, x):
        self.x, self.routing = x, moe.moe_route(self.shape, (x.float() @ self.router.float()).contiguous())
        y = moe.moe_fused_forward(self.shape, x, *self.w, self.routing, saved=self.stash)
        self.packed = moe.moe_saved_pack(self.shape, self.routing, self.stash)   # the stash is the next layer's now
        return x + y

    def backward(self, dy):
        moe.moe_saved_unpack(self.shape, self.routing, self.packed, self.stash)
        grads = moe.moe_fused_backward(self.shape, dy, self.x, *self.w, self.routing, self.stash)
        dlogits = moe.moe_route_backward(self.shape, self.routing, grads["dtopk_w"])
        grads["drouter"] = self.x.float().T @ dlogits
        return dy + grads["dx"] + (dlogits @ self.router.float().T).to(dy.dtype), grads


def main():
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--tokens", type=int, default=1000)
    args.add_argument("--layers", type=int, default=3)
    args = args.parse_args()
    T, d, E, k, I = args.tokens, 256, 16, 4, 192
    g = torch.Generator(device="cuda").manual_seed(0)
    stash = moe.alloc_saved(moe.make_shape(T, d, E, k, I), "cuda")
    layers = [RoutedLayer(T, d, E, k, I, stash, g) for _ in range(args.layers)]
    x = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    for one in layers:
        x = one.forward(x)
    kept = sum(one.packed.codes.numel() + one.packed.scales.numel() for one in layers)
    print(f"{args.layers} layers keep {kept / 1e6:.2f} MB, their stashes would be {args.layers * stash.numel() / 1e6:.2f} MB", flush=True)
    # the last layer: experts of one's own
    h = x.float().requires_grad_()
    w = (torch.randn((E, d, d), generator=g, device="cuda") * d ** -0.5).requires_grad_()
    routing = moe.moe_route(moe.make_shape(T, d, E, k, 64), torch.randn((T, E), generator=g, device="cuda"))
    loss = own_experts(h, routing, w).square().mean()
    loss.backward()
    dy = (h.grad * 1e3).to(torch.bfloat16)   # (a loss scale)
    for one in reversed(layers):
        dy, grads = one.backward(dy)
        print("gradients: " + ", ".join(f"{n} {float(v.float().norm()):.3e}" for n, v in grads.items()), flush=True)
    print(f"loss {float(loss.detach()):.5f}, gradient of the own experts {float(w.grad.norm()):.3e}")


if __name__ == "__main__":
    main()
