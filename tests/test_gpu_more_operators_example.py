"""The examples that run the 4-bit experts, the packed stash and experts of one's own as a user's program does."""
import sys
from pathlib import Path

import pytest
import torch

import paper_2604_19241_amd as moe

pytestmark = pytest.mark.gpu
sys.path.insert(0, str(Path(__file__).resolve().parents[1] / "examples"))


@pytest.mark.parametrize("T,kw", [(1, {}), (37, {}), (900, {}), (3000, dict(d=1408, I=1536, E=8, k=2)), (200, dict(d=200, I=104, E=20, k=6, e_start=5, e_count=10))])
def test_four_bit_experts(T, kw):
    import four_bit_experts as ex
    if kw.get("d") == 200:   # widths that moe_route's shape does not have: the operators by themselves
        layer, g = ex.layer(**kw)
        routing = moe.moe_route(moe.make_shape(T, 64, layer.E, layer.k, 64, layer.e_start, layer.e_count), torch.randn((T, layer.E), generator=g, device="cuda"))
        x = torch.randn((T, layer.d), generator=g, device="cuda").to(torch.bfloat16)
        o, _ = layer.experts(x, routing)
        y = moe.moe_combine_forward(moe.make_dispatch_shape(T, layer.k, layer.d), o, routing.inv_perm, routing.topk_w)
    else:
        layer, g = ex.layer(**kw)
        x, logits = ex.batch(layer, T, g)
        routing, y = layer.route(logits), layer.step(x, logits)
    want = ex.plain_step(layer, x, routing)
    # o and y are rounded to bf16 (at most 2^-8 of each value, by themselves below 0.6 % together); an h that lies between two steps may fall to the other side, one in 10^5
    assert float((y.double() - want).norm() / want.norm()) < 1e-2


def test_a_captured_serving_step():
    """The whole step in one graph, as a server replays it, with other tokens each time."""
    import four_bit_experts as ex
    layer, g = ex.layer()
    x, logits = ex.batch(layer, 64, g)
    layer.step(x, logits)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(x, logits)
    for _ in range(4):
        new_x, new_logits = ex.batch(layer, 64, g)
        x.copy_(new_x), logits.copy_(new_logits)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, layer.step(x, logits))


def test_two_streams_at_once():
    """Two servers' steps beside each other: the operators share nothing."""
    import four_bit_experts as ex
    sides = []
    for seed in (1, 2):
        layer, g = ex.layer(seed=seed)
        x, logits = ex.batch(layer, 300, g)
        sides.append((layer, x, logits, layer.step(x, logits)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    got = [[], []]
    for _ in range(10):
        for i, (layer, x, logits, _) in enumerate(sides):
            with torch.cuda.stream(streams[i]):
                got[i].append(layer.step(x, logits))
    torch.cuda.synchronize()
    for i, (_, _, _, want) in enumerate(sides):
        assert all(torch.equal(y, want) for y in got[i])


@pytest.mark.parametrize("T,e_start,e_count", [(50, 0, 8), (300, 2, 4)])
def test_experts_of_ones_own(T, e_start, e_count):
    """Autograd through dispatch and combine against torch's own in 64 bits."""
    import packed_stash_training as ex
    d, E, k = 64, 8, 3
    g = torch.Generator(device="cuda").manual_seed(T)
    routing = moe.moe_route(moe.make_shape(T, d, E, k, 64, e_start, e_count), torch.randn((T, E), generator=g, device="cuda"))
    x, w = torch.randn((T, d), generator=g, device="cuda"), torch.randn((e_count, d, d), generator=g, device="cuda") * d ** -0.5
    dy = torch.randn((T, d), generator=g, device="cuda")
    leaves = [v.clone().requires_grad_() for v in (x, w, routing.topk_w)]
    y = ex.own_experts(leaves[0], routing, leaves[1], leaves[2])
    got = torch.autograd.grad(y, leaves, dy)
    wide = [v.double().requires_grad_() for v in (x, w, routing.topk_w)]
    local = routing.inv_perm >= 0
    e = torch.where(local, routing.topk_idx - e_start, 0).long()
    out = torch.tanh(torch.stack([wide[0] @ wide[1][i] for i in range(e_count)], 1))   # [T, experts, d]
    want_y = (torch.take_along_dim(out, e[:, :, None], 1) * (wide[2] * local)[:, :, None]).sum(1)
    want = torch.autograd.grad(want_y, wide, dy.double())
    # fp32 throughout: sums of up to 64 and T k terms
    for a, b in zip([y, *got], [want_y, *want]):
        assert float((a.detach().double() - b.detach()).norm() / b.detach().norm()) < 1e-5
    assert (got[2][~local] == 0).all()


def test_layers_that_share_a_stash():
    import packed_stash_training as ex
    T, d, E, k, I = 200, 128, 8, 2, 192
    g = torch.Generator(device="cuda").manual_seed(3)
    stash = moe.alloc_saved(moe.make_shape(T, d, E, k, I), "cuda")
    layers = [ex.RoutedLayer(T, d, E, k, I, stash, g) for _ in range(3)]
    x = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    for one in layers:
        x = one.forward(x)
    dy = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    for one in reversed(layers):
        dx, grads = one.backward(dy)
        # the same backward pass from a stash of its own that holds the same packed values
        alone = moe.alloc_saved(one.shape, "cuda")
        want = moe.moe_fused_backward(one.shape, dy, one.x, *one.w, one.routing, moe.moe_saved_unpack(one.shape, one.routing, one.packed, alone))
        assert all(torch.equal(grads[n], want[n]) for n in want)
        assert torch.isfinite(dx).all() and torch.isfinite(grads["drouter"]).all()
        dy = dx
