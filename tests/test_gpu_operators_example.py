"""The example that runs the router's loss, the routed experts and the projections with adapters together."""
import sys
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, str(Path(__file__).resolve().parents[1] / "examples"))


@pytest.mark.parametrize("T", [100, 1500])
def test_a_step_of_the_layer(T):
    import adapter_router_step as ex
    layer = ex.Layer(T, 5, adapters=3)
    x, dy, ids, offsets, mask = ex.batch(T, 5, 3)
    before = {k: v.clone() for k, v in layer.shared.master.items()}
    out = layer.step(x, dy, ids, offsets, mask)
    for name, p, d in (("shared", layer.shared, dy), ("router", layer.router, out["dlogits"])):
        for key, want in zip(("da", "db"), ex.plain_factors(p, x, d, ids)):
            # two fp32 sums of up to 512 products and of up to 1500 tokens, and a pair of bf16 terms nowhere: fp32 roundings alone
            assert float((out[name][key].double() - want).norm() / want.norm()) < 1e-5, (name, key)
    # the logits' gradient: what the gates and the balance loss give by themselves, added
    import paper_2604_19241_amd as moe
    gates = moe.moe_route_backward(layer.experts, out["routing"], out["dtopk_w"])
    lse = torch.logsumexp(out["logits"].double(), 1)
    n = int(mask.sum())
    p = torch.exp(out["logits"].double() - lse[:, None]) * mask[:, None]
    want = gates.double()
    for a, b in zip(offsets.tolist(), offsets.tolist()[1:]):
        kept = mask[a:b]
        f = torch.bincount(out["routing"].topk_idx[a:b][kept].long().view(-1), minlength=32).double() / (4 * int(kept.sum()))
        want[a:b] += p[a:b] * (0.01 * 32 / n * (f - (p[a:b] @ f)[:, None]) + 0.001 * 2 / n * lse[a:b, None])
    assert ((out["dlogits"].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6 * want.abs().max()).all()
    layer.step(x, dy, ids, offsets, mask, rate=0.1)
    assert all(not torch.equal(before[k], v) for k, v in layer.shared.master.items())
