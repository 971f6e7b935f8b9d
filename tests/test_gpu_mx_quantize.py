"""Values into microscaled 4-bit floating point and back."""
import pytest
import torch

import mx_cases as mx
import paper_2604_19241_amd as moe
from helpers import say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def check(x):
    K = x.shape[1]
    q = moe.moe_mx_quantize(x)
    want, scales = mx.stand_for(x)
    assert q.codes.shape == (x.shape[0], mx.padded(K) // 2) and q.scales.shape == (x.shape[0], mx.padded(K) // 32)
    # (a block whose values are all zeros or too small for a scale has the smallest)
    assert torch.equal(q.scales, scales)
    assert mx.same(mx.values(q.codes, q.scales, K), want)
    assert (mx.nibbles(q.codes, mx.padded(K))[:, K:] % 8 == 0).all()   # the padding
    assert mx.same(moe.moe_mx_values(q), want) and mx.same(moe.moe_mx_values(q, out_dtype=F32), want)
    return q


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,K,pad", [(1, 8, 0), (1, 7168, 0), (3, 24, 8), (65, 32, 0), (64, 128, 64), (33, 136, 8), (700, 520, 0), (17, 1000, 24), (5, 1032, 0), (2, 65536, 0),
                                        (9000, 64, 0)])
def test_every_length(rows, K, pad, dtype):
    say(f"[mx] {rows} {K} {pad} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(rows + K)
    wide = torch.full((rows, K + pad), float("nan"), device="cuda")
    wide[:, :K] = torch.randn((rows, K), generator=g, device="cuda")
    check(wide.to(dtype)[:, :K])
    # magnitudes over all of the type's range, a block's within 2^8
    e = torch.randint(-130, 119, (rows, -(-K // 32), 1), generator=g, device="cuda").expand(-1, -1, 32).flatten(1)[:, :K] + torch.randint(0, 8, (rows, K), generator=g, device="cuda")
    wide[:, :K] = (wide[:, :K].double() * torch.exp2(e.double())).to(F32)
    check(wide.to(dtype)[:, :K])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_at_the_borders(dtype):
    ties = [0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.96875, 4.0]
    eps = torch.finfo(dtype).eps
    base = torch.tensor([s * v * (1 + n * eps) for v in ties for n in (-1, 0, 1) for s in (1, -1)])   # 72 values
    x = torch.zeros((6, 96))
    x[:, :72] = base
    x[:, 0] = x[:, 32] = x[:, 64] = 4.0    # every block's scale is 1
    x = x * torch.tensor([1.0, 2.0 ** -100, 2.0 ** 100, 2.0 ** 125, 2.0 ** -127, 3.0])[:, None]
    check(x.to(dtype).cuda())
    y = torch.zeros((8, 64))
    y[0, 3], y[1, 40], y[2, 63] = float("inf"), -float("inf"), float("nan")
    y[3] = 2.0 ** -133
    y[4] = 2.0 ** -126
    y[5] = 3.3895e38
    y[6, 31], y[6, 32] = 1e-30, 1e30   # neighbours of two blocks
    y[7] = -0.0
    check(y.to(dtype).cuda())


def test_every_code_and_scale_back():
    codes = (torch.arange(64, device="cuda") % 16 * 17).to(torch.uint8).expand(256, 64).contiguous()
    scales = torch.arange(256, device="cuda").to(torch.uint8)[:, None].expand(256, 4).contiguous()
    q = moe.MXTensor(codes, scales, 128)
    want = mx.values(codes, scales, 128)
    for dtype in (BF, F32):
        assert mx.same(moe.moe_mx_values(q, out_dtype=dtype), want.to(dtype).double())
    assert mx.same(moe.moe_mx_values(moe.MXTensor(codes, scales, 104)), want[:, :104].to(BF).double())


@pytest.mark.parametrize("E,K,N", [(1, 8, 8), (3, 128, 128), (2, 136, 72), (5, 264, 264), (1, 1000, 40), (2, 2048, 768), (4, 64, 1000), (1, 512, 65536)])
def test_weights(E, K, N):
    say(f"[mx] weights {E} {K} {N}")
    g = torch.Generator(device="cuda").manual_seed(K + N)
    w = (torch.randn((E, K, N), generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (E, K, N), generator=g, device="cuda").float())).to(BF)
    w[0, 0, N - 1] = float("nan")
    q = moe.moe_mx_quantize_weights(w)
    assert q.codes.shape == (E, N, mx.padded(K) // 2) and q.scales.shape == (E, N, mx.padded(K) // 32) and q.K == K
    for e in range(E):
        one = moe.moe_mx_quantize(w[e].T.contiguous())
        assert torch.equal(q.scales[e], one.scales) and mx.same(mx.values(q.codes[e], q.scales[e], K), mx.values(one.codes, one.scales, K))
    assert (mx.nibbles(q.codes, mx.padded(K))[..., K:] % 8 == 0).all()
    assert mx.same(moe.moe_mx_values(q), mx.values(q.codes, q.scales, K))


def test_no_rows_outputs_of_ones_own_and_long_tensors():
    q = moe.moe_mx_quantize(torch.empty((0, 64), dtype=BF, device="cuda"))
    assert q.codes.shape == (0, 64) and moe.moe_mx_values(q).shape == (0, 64)
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((40, 256), generator=g, device="cuda").to(BF)
    mine = moe.MXTensor(torch.empty((40, 128), dtype=torch.uint8, device="cuda"), torch.empty((40, 8), dtype=torch.uint8, device="cuda"), 256)
    q = moe.moe_mx_quantize(x, out=mine)
    assert q.codes is mine.codes and q.scales is mine.scales
    v = torch.empty((40, 256), device="cuda")
    assert moe.moe_mx_values(q, out_dtype=F32, out=v) is v and mx.same(v, mx.stand_for(x)[0])
    rows, K = (1 << 32) // 4096 + 3, 4096   # offsets beyond 32 bits
    say("[mx] large tensor")
    x = torch.zeros((rows, K), dtype=BF, device="cuda")
    x[-2:] = torch.randn((2, K), generator=g, device="cuda").to(BF)
    q = moe.moe_mx_quantize(x)
    assert mx.same(moe.moe_mx_values(q)[-2:], mx.stand_for(x[-2:])[0])


def test_streams_and_graphs():
    g = torch.Generator(device="cuda").manual_seed(0)
    src, w = torch.randn((300, 200), generator=g, device="cuda").to(BF), torch.randn((2, 136, 40), generator=g, device="cuda").to(BF)
    x = src.clone()

    def run():
        q, p = moe.moe_mx_quantize(x), moe.moe_mx_quantize_weights(w)
        return [q.codes, q.scales, moe.moe_mx_values(q), p.codes, p.scales]

    want = run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        x.zero_()
        torch.cuda._sleep(40_000_000)
        x.copy_(src)
        got = run()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for step in range(3):
        x.copy_(src * (step + 0.3))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        assert all(torch.equal(a, b) for a, b in zip(got, run())), step
