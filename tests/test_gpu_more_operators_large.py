"""More rows than one launch has, and buffers whose bytes are beyond 32 bits, in what the operators' own tests leave out: the last rows against the definitions."""
import pytest
import torch

import mx_cases as mx
import paper_2604_19241_amd as moe
from helpers import say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def normal(g, *sizes):
    return torch.randn(sizes, generator=g, device="cuda")


def test_more_tokens_than_a_launch_has():
    T, d = (1 << 24) + 5, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    shape = moe.make_dispatch_shape(T, 1, d)
    x, w = normal(g, T, d).to(BF), normal(g, T, 1)
    row_of = torch.arange(T - 1, -1, -1, device="cuda", dtype=torch.int32).view(T, 1)
    say("[large] dispatch, combine")
    xs = moe.moe_dispatch_forward(shape, x, row_of)
    assert torch.equal(xs, x.flip(0))
    assert torch.equal(moe.moe_dispatch_backward(shape, xs, row_of), x)
    want = (w * x.float()).to(BF)   # (one product in fp32, one rounding)
    assert torch.equal(moe.moe_combine_forward(shape, xs, row_of, w), want)
    got = moe.moe_combine_backward(shape, x, xs, row_of, w)
    assert torch.equal(got["do"], want.flip(0))
    dot = x.double().square().sum(1, keepdim=True)
    assert ((got["dw"] - dot).abs() <= 17 * 2.0 ** -24 * dot).all()   # eight products, nine additions


def test_more_rows_than_a_launch_has():
    rows, K = (1 << 24) + 5, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    x = normal(g, rows, K).to(BF)
    say("[large] quantize, values")
    v = moe.moe_mx_values(moe.moe_mx_quantize(x))
    for part in (slice(0, 9), slice(-9, None), slice((1 << 24) - 4, (1 << 24) + 4)):
        assert mx.same(v[part], mx.stand_for(x[part])[0])


@pytest.mark.parametrize("rows,K,N", [(70001, 128, 32768), (70001, 1280, 32768)])
def test_results_of_products_beyond_32_bits(rows, K, N):
    """Tiles of either size."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = normal(g, rows, K).to(BF)
    a = moe.moe_mx_quantize(x)
    w, u = (moe.moe_mx_quantize_weights((normal(g, 1, K, N) * K ** -0.5).to(BF)) for _ in range(2))
    offsets = torch.tensor([0, rows - 1], dtype=torch.int32, device="cuda")
    shape = moe.make_mx_shape(rows, K, N, 1)
    last = slice(rows - 6, rows - 1)
    av = mx.values(a.codes[last], a.scales[last], K)

    def sums(m):
        v = mx.values(m.codes[0], m.scales[0], K)
        return av @ v.T, (K / 64 + 18) * 2.0 ** -23 * (av.abs() @ v.abs().T)   # as for the small ones

    (gate, eg), (up, eu) = sums(w), sums(u)
    say(f"[large] product {rows} {K} {N}")
    y = torch.full((rows, N), 7.0, dtype=BF, device="cuda")
    moe.moe_mx_product(shape, a, w, offsets, y=y)
    assert ((y[last].double() - gate).abs() <= eg + 2.0 ** -8 * gate.abs()).all() and (y[-1] == 7.0).all()
    h = y.fill_(7.0)
    say(f"[large] gate and up {rows} {K} {N}")
    moe.moe_mx_gate_up(shape, a, w, u, offsets, h=h)
    s = torch.sigmoid(gate)
    want = gate * s * up
    err = 1.1 * up.abs() * eg + (gate * s).abs() * eu + 1.1 * eg * eu + ((gate.abs() + 8) * 2.0 ** -22 + 2.0 ** -8) * (want.abs() + 1.1 * up.abs() * eg)
    assert ((h[last].double() - want).abs() <= err + 1e-30).all() and (h[-1] == 7.0).all()
    q = moe.moe_mx_gate_up(shape, a, w, u, offsets, quantize=True)
    want = moe.moe_mx_quantize(h[last])
    assert torch.equal(q.codes[last], want.codes) and torch.equal(q.scales[last], want.scales)


def test_a_stash_beyond_32_bits():
    T, k, I = 1 << 17, 8, 2048
    g = torch.Generator(device="cuda").manual_seed(4)
    shape = moe.make_shape(T, 64, 8, k, I)
    routing = moe.moe_route(shape, normal(g, T, 8))
    assert int(routing.offsets[-1]) == T * k
    saved, other = moe.alloc_saved(shape, "cuda").zero_(), moe.alloc_saved(shape, "cuda").zero_()
    gu = moe.saved_views(shape, saved)["gu"]
    parts = [slice(0, 5), slice((1 << 31) // (4 * I) - 3, (1 << 31) // (4 * I) + 3), slice((1 << 32) // (4 * I) - 3, (1 << 32) // (4 * I) + 3), slice(T * k - 5, T * k)]
    for p in parts:
        gu[p] = normal(g, p.stop - p.start, 2 * I).to(BF)
    say("[large] pack, unpack")
    moe.moe_saved_unpack(shape, routing, moe.moe_saved_pack(shape, routing, saved), other)
    back = moe.saved_views(shape, other)
    for p in parts:
        v = gu[p].double().unflatten(-1, (-1, 32))
        step = torch.exp2(torch.floor(torch.log2(v.abs().amax(-1, keepdim=True))) - 6)
        v = ((v / step).round().clamp(-127, 127) * step).flatten(-2)
        assert torch.equal(back["gu"][p].double(), v)
        gate, up = v[:, :I], v[:, I:]
        h = gate * torch.sigmoid(gate) * up
        assert ((back["h"][p].double() - h).abs() <= (2.0 ** -8 + (gate.abs() + 8) * 2.0 ** -22) * h.abs() + 1e-30).all()
    assert int(torch.count_nonzero(back["gu"][5:1000])) == 0
