"""The stash in 8 bits: what comes back, and the backward pass from it, against the definitions in 64 bits."""
import pytest
import torch

import moe_synth
import paper_2604_19241_amd as moe
from helpers import say

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def stand_for(v):
    """The 8-bit values of blocks of 32 along the last axis, in 64 bits."""
    b = v.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -126)))
    step = torch.exp2(e - 6)
    q = ((b / step).round().clamp(-127, 127) * step)
    return torch.where(torch.isfinite(top), q, float("nan")).flatten(-2)


def routed(T, E, k, I, e_start=0, e_count=None, seed=0):
    shape = moe.make_shape(T, 64, E, k, I, e_start, e_count)
    g = torch.Generator(device="cuda").manual_seed(seed + T)
    return shape, moe.moe_route(shape, torch.randn((T, E), generator=g, device="cuda")), g


def check(shape, routing, gu):
    T, k, I = shape.T, shape.k, shape.I
    A = int(routing.offsets[-1])
    saved, other = moe.alloc_saved(shape, "cuda"), moe.alloc_saved(shape, "cuda")
    saved.fill_(0x5a), other.fill_(0x3c)
    moe.saved_views(shape, saved)["gu"][:A] = gu[:A]
    packed = moe.PackedSaved(torch.full((T * k, 2 * I), 77, dtype=torch.int8, device="cuda"), torch.full((T * k, I // 16), 99, dtype=torch.uint8, device="cuda"))
    moe.moe_saved_pack(shape, routing, saved, out=packed)
    assert (packed.codes[A:] == 77).all() and (packed.scales[A:] == 99).all()
    back = moe.saved_views(shape, moe.moe_saved_unpack(shape, routing, packed, other))
    want = stand_for(gu[:A])
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(back["gu"][:A]), nan)
    assert torch.equal(torch.where(nan, 0.0, back["gu"][:A].double()), torch.where(nan, 0.0, want))
    g, u = want[:, :I], want[:, I:]
    h = g * torch.sigmoid(g) * u
    # bf16's half step; the exponential's argument is rounded and its result off by about (|g| + 4) 2^-23 of itself, the reciprocal and two products by a step each; beyond 2^-126
    # and where the exponential overflows what is lost is below 2^-120 of the operands
    err = (2.0 ** -8 + (g.abs() + 8) * 2.0 ** -22) * h.abs() + 2.0 ** -120 * (1 + (g * u).abs())
    fine = torch.isfinite(h) & (h.abs() < 3.3e38)
    assert ((back["h"][:A].double() - h).abs()[fine] <= err[fine]).all()
    assert torch.equal(torch.isnan(back["h"][:A]), torch.isnan(h))
    # rows behind the last one, and the part that the backward pass does not read, as they were
    raw = other.clone()
    views = moe.saved_views(shape, raw)
    views["gu"][:A] = 0
    views["h"][:A] = 0
    fresh = torch.full_like(raw, 0x3c)
    views = moe.saved_views(shape, fresh)
    views["gu"][:A] = 0
    views["h"][:A] = 0
    assert torch.equal(raw, fresh)
    return packed


@pytest.mark.parametrize("T,E,k,I,e_start,e_count", [(1, 8, 1, 64, 0, 8), (1, 8, 8, 192, 2, 3), (33, 8, 2, 64, 0, 8), (257, 64, 6, 1408, 0, 64), (300, 16, 4, 704, 4, 5),
                                                     (1000, 8, 2, 1024, 0, 8), (5, 8, 2, 14336, 0, 8), (600, 16, 16, 128, 0, 1)])
def test_what_comes_back(T, E, k, I, e_start, e_count):
    say(f"[saved] {T} {E} {k} {I} {e_start} {e_count}")
    shape, routing, g = routed(T, E, k, I, e_start, e_count)
    gu = torch.randn((T * k, 2 * I), generator=g, device="cuda")
    check(shape, routing, (gu * 3).to(BF))
    # magnitudes over all of the type's range, a block's within 2^8
    e = torch.randint(-130, 118, (T * k, 2 * I // 32, 1), generator=g, device="cuda").expand(-1, -1, 32) + torch.randint(0, 8, (T * k, 2 * I // 32, 32), generator=g, device="cuda")
    check(shape, routing, (gu.double() * torch.exp2(e.flatten(1).double())).to(BF))


def test_values_at_the_borders():
    shape, routing, g = routed(64, 8, 1, 64)
    gu = torch.zeros((64, 128), device="cuda")
    for r in range(40):   # largest values around a power of two and at 127.5 steps; ties; signs
        top = [1.0, 1.9921875, 1.984375, 1.9765625, 0.99609375, 1.0078125, -1.9921875, -1.0][r % 8]
        gu[r] = torch.arange(128, device="cuda") % 32 * (top / 64)
        gu[r, ::32] = top
        gu[r] *= 2.0 ** (r - 20)
    gu[40] = 2.0 ** -133
    gu[41] = torch.where(torch.arange(128, device="cuda") % 2 == 0, 3.3895e38, -1.0)
    gu[42, 5] = float("inf")
    gu[43, 70] = -float("inf")
    gu[44, 127] = float("nan")
    gu[45] = 2.0 ** -126
    gu[46] = 1.99 * 2.0 ** -127
    check(shape, routing, gu.to(BF))


def test_no_tokens_and_no_rows():
    shape, routing, _ = routed(0, 8, 2, 64)
    saved = moe.alloc_saved(shape, "cuda")
    packed = moe.moe_saved_pack(shape, routing, saved)
    assert packed.codes.shape == (0, 128) and moe.moe_saved_unpack(shape, routing, packed, saved) is saved
    shape = moe.make_shape(5, 64, 8, 2, 64, 6, 2)
    logits = torch.zeros((5, 8), device="cuda")
    logits[:, :2] = 1.0
    routing = moe.moe_route(shape, logits)
    assert int(routing.offsets[-1]) == 0
    check(shape, routing, torch.zeros((10, 128), dtype=BF, device="cuda"))


@pytest.mark.parametrize("T,E,k,e_start,e_count", [(300, 8, 2, 0, 8), (130, 16, 4, 3, 6)])
def test_the_backward_pass_from_it(T, E, k, e_start, e_count):
    """Two layers that share one stash: each one's gradients are those of its own packed activations."""
    say(f"[saved] backward {T} {E} {k}")
    d, I = 128, 192
    cfg = moe_synth.small_config(T=T, d=d, E=E, k=k, I=I, e_start=e_start, e_count=e_count)
    shape = moe.make_shape(**cfg.shape_dict())
    stash, layers = moe.alloc_saved(shape, "cuda"), []
    for seed in (1, 2):
        inp = {n: v.cuda() for n, v in moe_synth.make_inputs(cfg, seed=seed).items()}
        routing = moe.moe_route(shape, inp["logits"])
        moe.moe_fused_forward(shape, inp["x"], inp["w_gate"], inp["w_up"], inp["w_down"], routing, saved=stash)
        gu = moe.saved_views(shape, stash)["gu"].clone()
        layers.append((inp, routing, moe.moe_saved_pack(shape, routing, stash), gu))
    for inp, routing, packed, gu in reversed(layers):
        moe.moe_saved_unpack(shape, routing, packed, stash)
        got = moe.moe_fused_backward(shape, inp["dy"], inp["x"], inp["w_gate"], inp["w_up"], inp["w_down"], routing, stash)
        A = int(routing.offsets[-1])
        x, dy, wg, wu, wd = (inp[n].double() for n in ("x", "dy", "w_gate", "w_up", "w_down"))
        token, slot = routing.perm[:A].long() // k, routing.perm[:A].long()
        v = stand_for(gu[:A])
        g, u = v[:, :I], v[:, I:]
        sg = torch.sigmoid(g)
        h = g * sg * u
        want = {"dx": torch.zeros_like(x), "dw_gate": torch.zeros_like(wg), "dw_up": torch.zeros_like(wu), "dw_down": torch.zeros_like(wd),
                "dtopk_w": torch.zeros((T, k), dtype=torch.float64, device="cuda")}
        at = routing.offsets.tolist()
        for e in range(e_count):
            r = slice(at[e], at[e + 1])
            do = routing.topk_w.view(-1)[slot[r]].double()[:, None] * dy[token[r]]
            dh = do @ wd[e].T
            dg, du = dh * u[r] * sg[r] * (1 + g[r] * (1 - sg[r])), dh * g[r] * sg[r]
            want["dw_down"][e] = h[r].T @ do
            want["dw_gate"][e], want["dw_up"][e] = x[token[r]].T @ dg, x[token[r]].T @ du
            want["dx"].index_add_(0, token[r], dg @ wg[e].T + du @ wu[e].T)
            want["dtopk_w"].view(-1)[slot[r]] = ((dy[token[r]] @ wd[e].T) * h[r]).sum(1)
        for name, w in want.items():
            off = float((got[name].double() - w).norm() / w.norm())
            say(f"[saved] {name} {off:.1e}")
            # the bound of the fused backward pass: intermediate results in bf16 (dO, h, dG, dU, dXp), the result's rounding
            assert off <= 1e-2, name


def test_streams_and_graphs():
    shape, routing, g = routed(200, 8, 2, 128)
    saved, other = moe.alloc_saved(shape, "cuda"), moe.alloc_saved(shape, "cuda")
    other.zero_()
    gu = moe.saved_views(shape, saved)["gu"]
    src = torch.randn(gu.shape, generator=g, device="cuda").to(BF)

    def run():
        moe.moe_saved_unpack(shape, routing, moe.moe_saved_pack(shape, routing, saved), other)
        return [v.clone() for n, v in moe.saved_views(shape, other).items() if n != "o"]

    gu.copy_(src)
    want = run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        gu.zero_()
        torch.cuda._sleep(40_000_000)
        gu.copy_(src)
        got = run()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for step in range(3):
        gu.copy_(src * (step + 0.7))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        assert all(torch.equal(a, b) for a, b in zip(got, run())), step
