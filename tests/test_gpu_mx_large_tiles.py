"""Products in 4 bits in tiles of 256 x 256: the shortest reductions that are done in them, other streams and graphs; which kernel a shape takes is read from a captured graph."""
import ctypes

import pytest
import torch

import paper_2604_19241_amd as moe
from helpers import say
from test_gpu_launches import launches
from test_gpu_mx_product import check_gate_up, check_product, make

pytestmark = pytest.mark.gpu
F32 = torch.float32


def in_large_tiles(s):
    """The product's kernel, or gate and up's, is the one of 256 x 256 for this shape (any aligned address will do for kernels that never run)."""
    p, lib, shape = ctypes.c_void_p(4096), moe.load_library(), ctypes.byref(s["shape"])
    head = (shape, p, p, ctypes.c_int64(1 << 20), p, 1, p, p)
    if "u" in s:
        got = launches(lambda st: lib.moe_mx_gate_up(*head, p, p, p, p, None, None, st))
    else:
        got = launches(lambda st: lib.moe_mx_product(*head, p, p, 0, st))
    assert len(got) == 1, got
    return "mx_big_kernel" in got[0][0]


# 4 and 5 blocks of 128 values: two stages that are both requested at the beginning; two and a half, where the half one is the only one that is requested later.  K' = K or filled up.
@pytest.mark.parametrize("counts", [[6000], [6000, 1, 33]])
@pytest.mark.parametrize("K", [392, 512, 520, 640])
def test_the_shortest_reductions(counts, K):
    say(f"[mx large] {counts} {K}")
    s = make(counts, K, 65536)
    assert in_large_tiles(s)
    check_product(s)
    del s
    s = make(counts, K, 65528, tokens=900, k=3, spare=5, pair=True)
    assert in_large_tiles(s)
    check_gate_up(s)


def test_streams_graphs_and_runs():
    counts, N = [600, 130, 270], 15880
    say(f"[mx large] streams and graphs, {counts} {N}")
    s, one = make(counts, 4096, N, tokens=700, k=2, pair=True), make(counts, 4096, N)
    assert in_large_tiles(s) and in_large_tiles(one)
    src = s["a"].scales.clone()

    def run():
        y = moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"], perm=s["perm"], k=2, out_dtype=F32)
        q = moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], perm=s["perm"], k=2, quantize=True)
        return [y, q.codes, q.scales]

    want = run()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        s["a"].scales.zero_()
        torch.cuda._sleep(40_000_000)
        s["a"].scales.copy_(src)
        got = run()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for step in range(3):
        s["a"].scales.copy_(src + step)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        assert all(torch.equal(a, b) for a, b in zip(got, run())), step
