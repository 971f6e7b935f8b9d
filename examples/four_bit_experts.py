"""A MoE layer served with its experts in microscaled 4 bits.

    python examples/four_bit_experts.py [--tokens 37] [--steps 3] [--check]

The weights are quantised once.  A step routes its tokens, quantises them, multiplies each with its experts' gate and up projections (SwiGLU and the next quantisation in the same launch)
and with their down projections, and adds the experts' outputs with the gates' weights.  --check compares a step with plain torch operations in 64 bits on the same quantised values.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
import paper_2604_19241_amd as moe  # noqa: E402


class FourBitExperts:
    """The local experts [e_start, e_start + e_count) of a layer; w_gate, w_up [e_count,d,I] and w_down [e_count,I,d] bf16, as moe_fused_forward takes them."""

    def __init__(self, w_gate, w_up, w_down, E, k, e_start=0):
        self.e_count, self.d, self.I = w_gate.shape
        self.E, self.k, self.e_start = E, k, e_start
        self.w_gate, self.w_up, self.w_down = (moe.moe_mx_quantize_weights(w) for w in (w_gate, w_up, w_down))

    def route(self, logits):
        return moe.moe_route(moe.make_shape(logits.shape[0], self.d, self.E, self.k, self.I, self.e_start, self.e_count), logits)

    def experts(self, x, routing):
        """Rows of the experts' outputs [T k, d], in the routing's order."""
        rows = x.shape[0] * self.k
        up, down = moe.make_mx_shape(rows, self.d, self.I, self.e_count), moe.make_mx_shape(rows, self.I, self.d, self.e_count)
        h = moe.moe_mx_gate_up(up, moe.moe_mx_quantize(x), self.w_gate, self.w_up, routing.offsets, perm=routing.perm, k=self.k, quantize=True)
        return moe.moe_mx_product(down, h, self.w_down, routing.offsets), h

    def step(self, x, logits):
        routing = self.route(logits)
        o, _ = self.experts(x, routing)
        return moe.moe_combine_forward(moe.make_dispatch_shape(x.shape[0], self.k, self.d), o, routing.inv_perm, routing.topk_w)


def layer(d=512, I=256, E=32, k=4, e_start=0, e_count=None, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = E if e_count is None else e_count

    def normal(*s):
        return (torch.randn(s, generator=g, device="cuda") * s[1] ** -0.5).to(torch.bfloat16)

    return FourBitExperts(normal(n, d, I), normal(n, d, I), normal(n, I, d), E, k, e_start), g


def batch(layer, T, g):
    return torch.randn((T, layer.d), generator=g, device="cuda").to(torch.bfloat16), torch.randn((T, layer.E), generator=g, device="cuda")


def plain_step(layer, x, routing):
    """The same in 64 bits from the quantised activations and weights; h is rounded to bf16 and quantised by the library, as its values are the next product's inputs."""
    wide = lambda m: moe.moe_mx_values(m, out_dtype=torch.float32).double()  # noqa: E731
    a, wg, wu, wd = (wide(m) for m in (moe.moe_mx_quantize(x), layer.w_gate, layer.w_up, layer.w_down))
    y = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    at = routing.offsets.tolist()
    for e in range(layer.e_count):
        slots = routing.perm[at[e]:at[e + 1]].long()
        if slots.numel() == 0:
            continue
        t = slots // layer.k
        gate = a[t] @ wg[e].T
        h = (gate * torch.sigmoid(gate) * (a[t] @ wu[e].T)).to(torch.bfloat16)
        y.index_add_(0, t, routing.topk_w.view(-1)[slots].double()[:, None] * (wide(moe.moe_mx_quantize(h)) @ wd[e].T))
    return y


def main():
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--tokens", type=int, default=37)
    args.add_argument("--steps", type=int, default=3)
    args.add_argument("--check", action="store_true")
    args = args.parse_args()
    experts, g = layer()
    for step in range(args.steps):
        x, logits = batch(experts, args.tokens, g)
        y = experts.step(x, logits)
        if args.check:
            want = plain_step(experts, x, experts.route(logits))
            off = float((y.double() - want).norm() / want.norm())
            print(f"step {step}: relative error {off:.1e}")
            assert off < 1e-2
        print(f"step {step}: {args.tokens} tokens, output of {float(y.float().square().mean().sqrt()):.4f} rms", flush=True)


if __name__ == "__main__":
    main()
