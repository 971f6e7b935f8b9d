"""A fine-tuning step of one MoE layer: a router with its balance loss, routed experts, and a shared projection with a low-rank adapter
for every request of the packed batch.

    python examples/adapter_router_step.py [--tokens 4099] [--steps 3] [--check]

Every request (a run of tokens) has one of a few adapters, or none; the router's projection and the shared projection both have them.  The
step returns the losses and updates the adapters' factors; the projections and the experts stay as they are.  --check compares the adapters'
gradients of one step with those of plain torch operations in 64 bits.
"""
import argparse
import random
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
import paper_2604_19241_amd as moe  # noqa: E402


class Projection:
    """x W + s (x A^T) B with a pair of factors for every adapter; the factors are kept in fp32 and used in bf16."""

    def __init__(self, T, K, N, rank, adapters, out_dtype, g):
        self.shape, self.out_dtype = moe.make_adapter_shape(T, K, N, rank, adapters), out_dtype
        self.w = (torch.randn((K, N), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)
        self.master = {"a": torch.randn((adapters, rank, K), generator=g, device="cuda") * K ** -0.5,
                       "b": torch.randn((adapters, rank, N), generator=g, device="cuda") * 0.02}
        self.scale = torch.full((adapters,), 2.0, device="cuda")
        self.h = torch.empty((T, rank), device="cuda")
        self.ws = torch.empty(moe.moe_adapter_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")
        self.cast()

    def cast(self):
        self.a, self.b = (self.master[k].to(torch.bfloat16) for k in ("a", "b"))

    def forward(self, x, plan):
        return moe.moe_adapter_forward(self.shape, x, self.w, self.a, self.b, plan, scale=self.scale, out_dtype=self.out_dtype, h=self.h, ws=self.ws)

    def backward(self, dy, x, plan):
        return moe.moe_adapter_backward(self.shape, dy, x, self.w, self.a, self.b, plan, self.h, scale=self.scale, ws=self.ws)

    def update(self, grads, rate):
        self.master["a"].sub_(grads["da"], alpha=rate)
        self.master["b"].sub_(grads["db"], alpha=rate)
        self.cast()


class Layer:
    def __init__(self, T, seqs, d=512, E=32, k=4, I=256, rank=16, adapters=4, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.router = Projection(T, d, E, 8, adapters, torch.float32, g)
        self.shared = Projection(T, d, d, rank, adapters, torch.bfloat16, g)
        self.experts = moe.make_shape(T=T, d=d, E=E, k=k, I=I)
        self.balance = moe.make_balance_shape(T, E, k, seqs, balance_coef=0.01, z_coef=0.001)
        normal = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.05).to(torch.bfloat16)  # noqa: E731
        self.w = [normal(E, d, I), normal(E, d, I), normal(E, I, d)]

    def step(self, x, dy, ids, seq_offsets, mask, rate=0.0):
        """Forward, backward and (rate > 0) update for the gradient dy of the layer's output y = routed experts + shared projection."""
        plan = moe.moe_adapter_plan(self.shared.shape, ids)   # one for both projections
        logits = self.router.forward(x, plan)
        routing = moe.moe_route(self.experts, logits)
        stats = moe.moe_balance_forward(self.balance, logits, routing.topk_idx, seq_offsets=seq_offsets, mask=mask)
        saved = moe.alloc_saved(self.experts, x.device)
        y = moe.moe_fused_forward(self.experts, x, *self.w, routing, saved=saved) + self.shared.forward(x, plan)
        routed = moe.moe_fused_backward(self.experts, dy, x, *self.w, routing, saved)
        dlogits = moe.moe_balance_backward(self.balance, logits, routing.topk_idx, stats, torch.ones(1, device=x.device), seq_offsets=seq_offsets,
                                           topk_w=routing.topk_w, dtopk_w=routed["dtopk_w"], out_dtype=torch.bfloat16)
        shared, router = self.shared.backward(dy, x, plan), self.router.backward(dlogits, x, plan)
        if rate:
            self.shared.update(shared, rate)
            self.router.update(router, rate)
        dx = routed["dx"].float() + shared["dx"].float() + router["dx"].float()
        return {"y": y, "dx": dx, "loss": stats.loss, "counts": stats.counts, "logits": logits, "routing": routing, "dtopk_w": routed["dtopk_w"],
                "dlogits": dlogits, "shared": shared, "router": router}


def batch(T, seqs, adapters, d=512, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    cuts = [0] + sorted(rng.sample(range(1, T), seqs - 1)) + [T]
    ids = torch.empty(T, dtype=torch.int32)
    mask = torch.ones(T, dtype=torch.bool)
    for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
        ids[a:b] = i % (adapters + 1) - 1          # the first request has none
        mask[b - (b - a) // 10:b] = False          # padding at its end
    x, dy = ((torch.randn((T, d), generator=g, device="cuda") * s).to(torch.bfloat16) for s in (1.0, 0.1))
    return x, dy, ids.cuda(), torch.tensor(cuts, dtype=torch.int32, device="cuda"), mask.cuda()


def plain_factors(p, x, dy, ids):
    """Gradients of the factors, in 64 bits."""
    x, dy, a, b = x.double(), dy.double(), p.a.double(), p.b.double()
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for i in range(a.shape[0]):
        t = ids == i
        da[i] = p.scale[i].double() * (dy[t] @ b[i].T).T @ x[t]
        db[i] = p.scale[i].double() * (x[t] @ a[i].T).T @ dy[t]
    return da, db


def main():
    args = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    args.add_argument("--tokens", type=int, default=4099)
    args.add_argument("--steps", type=int, default=3)
    args.add_argument("--check", action="store_true")
    args = args.parse_args()
    seqs, adapters = 9, 4
    layer = Layer(args.tokens, seqs, adapters=adapters)
    x, dy, ids, offsets, mask = batch(args.tokens, seqs, adapters)
    for step in range(args.steps):
        if args.check and step == 0:
            out = layer.step(x, dy, ids, offsets, mask)
            for name, p, d in (("shared", layer.shared, dy), ("router", layer.router, out["dlogits"])):
                for key, want in zip(("da", "db"), plain_factors(p, x, d, ids)):
                    off = float((out[name][key].double() - want).norm() / want.norm())
                    print(f"{name} {key}: relative error {off:.1e}")
                    assert off < 1e-5
        out = layer.step(x, dy, ids, offsets, mask, rate=1e-2)
        loss, balance, z = out["loss"].tolist()
        print(f"step {step}: loss {loss:.5f} (balance {balance:.4f}, z {z:.4f}), busiest expert {int(out['counts'].sum(0).max())} slots", flush=True)


if __name__ == "__main__":
    main()
