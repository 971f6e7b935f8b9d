"""Products of rows sorted by expert with their experts' weights, in microscaled 4 bits, against the definition in 64 bits."""
import pytest
import torch

import mx_cases as mx
import paper_2604_19241_amd as moe
from helpers import say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
KEEP = 7.0


def random_mx(g, *sizes, spread=3):
    """Codes of every kind, scales around one, the padding zeros."""
    K = sizes[-1]
    lead, Kp = sizes[:-1], mx.padded(sizes[-1])
    c = torch.randint(0, 16, (*lead, Kp), generator=g, device="cuda", dtype=torch.uint8)
    c[..., K:] = 0
    s = torch.randint(127 - spread, 128 + spread, (*lead, Kp // 32), generator=g, device="cuda", dtype=torch.uint8)
    return moe.MXTensor(c[..., 0::2] + 16 * c[..., 1::2], s, K)


def make(counts, K, N, spare=0, tokens=None, k=1, seed=0, pair=False):
    g = torch.Generator(device="cuda").manual_seed(seed + K + N + sum(counts))
    E, A = len(counts), sum(counts)
    s = {"E": E, "A": A, "rows": A + spare, "K": K, "N": N, "k": k}
    s["offsets"] = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    s["perm"] = None
    if tokens is not None:
        s["perm"] = torch.full((A + spare,), -1, dtype=torch.int32, device="cuda")
        s["perm"][:A] = torch.randint(0, tokens * k, (A,), generator=g, device="cuda", dtype=torch.int32)
    s["a"] = random_mx(g, A + spare if tokens is None else tokens, K)
    s["w"] = random_mx(g, E, N, K)
    if pair:
        # gates of a size that silu bends
        s["w"] = moe.MXTensor(s["w"].codes, (s["w"].scales.int() - 3 - (K.bit_length() >> 1)).to(torch.uint8), K)
        s["u"] = random_mx(g, E, N, K)
    s["shape"] = moe.make_mx_shape(A + spare, K, N, E)
    return s


def wide(m):
    return mx.values(m.codes, m.scales, m.K)


def sums(s, name):
    """The products of every row with its expert's weights in 64 bits, and the sums of magnitudes."""
    a = wide(s["a"])
    a = a[s["perm"][:s["A"]].long() // s["k"]] if s["perm"] is not None else a[:s["A"]]
    v = torch.empty((s["A"], s["N"]), dtype=torch.float64, device="cuda")
    m = torch.empty_like(v)
    at = s["offsets"].tolist()
    for e in range(s["E"]):
        lo, hi = at[e], at[e + 1]
        if hi > lo:
            w = mx.values(s[name].codes[e], s[name].scales[e], s["K"])
            v[lo:hi], m[lo:hi] = a[lo:hi] @ w.T, a[lo:hi].abs() @ w.abs().T
    return v, m


def fp32_sum(s, m):
    """An instruction adds 64 products to the sum with one rounding, at worst half a step of 2^-23 of the magnitudes; sums of several parts join in up to 16 more.  Twice that, as
    the order inside an instruction is the hardware's."""
    return (s["K"] / 64 + 18) * 2.0 ** -23 * m


def near(got, want, err, what):
    off = (got.double() - want).abs()
    assert (off <= err + 1e-30).all(), (what, float((off - err).max()), torch.nonzero(off > err)[:4].tolist())


def check_product(s):
    for dtype in (BF, F32):
        y = torch.full((s["rows"], s["N"]), KEEP, dtype=dtype, device="cuda")
        got = moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"], perm=s["perm"], k=s["k"], out_dtype=dtype, y=y)
        assert got is y
        v, m = sums(s, "w")
        near(y[:s["A"]], v, fp32_sum(s, m) + (2.0 ** -8 if dtype is BF else 0.0) * v.abs(), dtype)
        assert (y[s["A"]:] == KEEP).all()


def check_gate_up(s):
    h = torch.full((s["rows"], s["N"]), KEEP, dtype=BF, device="cuda")
    moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], perm=s["perm"], k=s["k"], h=h)
    (g, mg), (u, mu) = sums(s, "w"), sums(s, "u")
    sg = torch.sigmoid(g)
    want = g * sg * u
    eg, eu = fp32_sum(s, mg), fp32_sum(s, mu)
    # the sums' errors (silu's slope is below 1.1), the exponential of a rounded argument, the reciprocal and the products, bf16's rounding
    err = 1.1 * u.abs() * eg + (g * sg).abs() * eu + 1.1 * eg * eu + ((g.abs() + 8) * 2.0 ** -22 + 2.0 ** -8) * (want.abs() + 1.1 * u.abs() * eg)
    near(h[:s["A"]], want, err, "h")
    assert (h[s["A"]:] == KEEP).all()
    out = moe.MXTensor(torch.full((s["rows"], mx.padded(s["N"]) // 2), 0x77, dtype=torch.uint8, device="cuda"),
                       torch.full((s["rows"], mx.padded(s["N"]) // 32), 0x55, dtype=torch.uint8, device="cuda"), s["N"])
    q = moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], perm=s["perm"], k=s["k"], quantize=True, h=out)
    assert q.codes is out.codes and q.K == s["N"]
    want = moe.moe_mx_quantize(h[:s["A"]])
    assert torch.equal(q.scales[:s["A"]], want.scales) and torch.equal(q.codes[:s["A"]], want.codes)
    assert (q.codes[s["A"]:] == 0x77).all() and (q.scales[s["A"]:] == 0x55).all()


COUNTS = [0, 1, 2, 31, 32, 33, 0, 63, 64, 65, 96, 127, 128, 129, 200, 300, 0]


@pytest.mark.parametrize("K,N", [(8, 8), (64, 72), (128, 256), (136, 264), (256, 128), (384, 520), (520, 136), (640, 32), (1024, 96), (2048, 768), (7168, 40), (896, 1000)])
def test_widths(K, N):
    say(f"[mx product] {K} {N}")
    check_product(make(COUNTS, K, N, spare=5))
    check_gate_up(make(COUNTS, K, N, spare=3, pair=True))


@pytest.mark.parametrize("counts", [[1], [8], [0, 0, 5, 0], [1] * 8, [0] * 40 + [3] + [0] * 100, [1, 0] * 32, [2] * 65, [5, 0, 40, 0] * 50, [700], [1] * 1024, [0] * 1000 + [140, 3], [33] * 128,
                                    [2000, 1, 1, 1], [16] * 10 + [17] * 10, [4, 5, 8, 9]])
def test_experts_of_any_number_and_size(counts):
    say(f"[mx product] {len(counts)} experts, {sum(counts)} rows")
    N = 136 if len(counts) > 200 else 264
    check_product(make(counts, 384, N, tokens=30, k=4, spare=7))
    check_gate_up(make(counts, 384, N, tokens=30, k=4, pair=True))


@pytest.mark.parametrize("K,N", [(1280, 256), (1288, 264), (1408, 520), (2048, 136), (1544, 40), (4096, 128)])
@pytest.mark.parametrize("counts", [[300, 5, 0, 257, 256, 64, 33, 1], [1000], [0, 97, 0, 230, 1], [191, 193, 512, 31, 224], [100] * 70])
def test_many_rows_and_long_reductions(counts, K, N):
    """Full tiles and parts of them, in an odd and an even number of 128 values."""
    say(f"[mx product] {len(counts)} experts, {sum(counts)} rows, {K} {N}")
    check_product(make(counts, K, N, spare=3))
    check_gate_up(make(counts, K, N, tokens=77, k=2, pair=True))


@pytest.mark.parametrize("counts", [[16] * 12, [16] * 11 + [17], [3, 9, 0, 16], [20, 4, 0, 31], [32, 33]])
@pytest.mark.parametrize("K,N", [(4096, 264), (4224, 1000), (512, 72)])
def test_few_rows(counts, K, N):
    """Narrow tiles, for all experts or for some: by the rows of the largest, the reduction and how many wide ones there would be."""
    say(f"[mx product] {counts} {K} {N}")
    check_product(make(counts, K, N, tokens=11, k=3))
    check_gate_up(make(counts, K, N, spare=1, pair=True))


@pytest.mark.parametrize("T,K,N,E,k,e_start,e_count", [(1, 768, 2048, 128, 8, 0, 128), (37, 7168, 256, 256, 8, 32, 32), (300, 512, 1024, 8, 2, 0, 8), (2000, 1024, 384, 128, 6, 0, 128)])
def test_with_a_routing(T, K, N, E, k, e_start, e_count):
    say(f"[mx product] {T} {K} {N} {E} {k}")
    g = torch.Generator(device="cuda").manual_seed(T)
    r = moe.moe_route(moe.make_shape(T, 64, E, k, 64, e_start, e_count), torch.randn((T, E), generator=g, device="cuda"))
    s = make(r.counts.tolist(), K, N, spare=T * k - int(r.offsets[-1]), tokens=T, k=k, pair=True)
    s["offsets"], s["perm"] = r.offsets, r.perm
    check_product(s)
    check_gate_up(s)


def test_no_rows():
    s = make([0, 0, 0], 128, 64, spare=9, pair=True)
    check_product(s)
    check_gate_up(s)
    s = make([0, 0, 0], 128, 64, pair=True)
    assert moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"]).shape == (0, 64)
    assert moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], quantize=True).codes.shape == (0, 64)


@pytest.mark.parametrize("counts", [[3, 40, 150], [1, 2, 3], [300, 0, 200]])
def test_values_that_are_not_numbers_stay_where_they_are(counts):
    s = make(counts, 512, 136, pair=True, seed=4)
    clean = moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"])
    clean_h = moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"])
    row, expert, col = counts[0] + 1, 2, 77
    s["a"].scales[row, 5] = 255
    s["w"].scales[expert, col, 3] = 255
    y = moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"])
    h = moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"])
    bad = torch.zeros(clean.shape, dtype=torch.bool, device="cuda")
    bad[row] = True
    bad[sum(counts[:2]):, col] = True
    for got, want in ((y, clean), (h, clean_h)):
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])
    q = moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], quantize=True)
    want = moe.moe_mx_quantize(h)
    assert torch.equal(q.scales, want.scales) and torch.equal(q.codes, want.codes)


def test_scales_at_the_ends_of_their_range():
    s = make([3, 40, 150], 256, 72, seed=5)
    s["a"].scales[:, 0], s["a"].scales[:, 1] = 254, 0
    s["w"].scales[:, :, 0], s["w"].scales[:, :, 1] = 0, 254
    check_product(s)   # (values around 2^127 by values around 2^-127)


def test_routings_that_do_not_fit_reach_no_memory_outside():
    """Offsets beyond the buffer and sources beyond the tokens: rows of unspecified values, everything else as it should be."""
    s = make([10, 20, 30], 128, 64, tokens=9, k=2, spare=4)
    s["perm"][3], s["perm"][4], s["perm"][59] = -5, 2 ** 31 - 1, 18
    y = moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"], perm=s["perm"], k=2)
    s["perm"][3], s["perm"][4], s["perm"][59] = 0, 0, 0
    want = moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"], perm=s["perm"], k=2)
    fine = [r for r in range(60) if r not in (3, 4, 59)]
    assert torch.equal(y[fine], want[fine])
    wild = torch.tensor([0, 10, 30, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    y = moe.moe_mx_product(s["shape"], s["a"], s["w"], wild, perm=s["perm"].clamp(min=0), k=2)
    assert torch.equal(y[:60], want[:60])
    wild = torch.tensor([-7, 10, 30, 5], dtype=torch.int32, device="cuda")
    y = moe.moe_mx_product(s["shape"], s["a"], s["w"], wild, perm=s["perm"], k=2)
    assert torch.equal(y[:30], want[:30])


def test_streams_graphs_and_runs():
    s = make(COUNTS, 640, 264, tokens=50, k=3, pair=True)
    src = s["a"].scales.clone()
    y = torch.zeros((s["rows"], s["N"]), device="cuda")

    def run():
        moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"], perm=s["perm"], k=3, out_dtype=F32, y=y)
        q = moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], perm=s["perm"], k=3, quantize=True)
        return [y.clone(), q.codes, q.scales]

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


def test_offsets_beyond_32_bits():
    """Weights and activations whose last bytes lie beyond 2^32."""
    E, N, K = 40, 16384, 16384
    g = torch.Generator(device="cuda").manual_seed(1)
    w = moe.MXTensor(torch.zeros((E, N, K // 2), dtype=torch.uint8, device="cuda"), torch.full((E, N, K // 32), 127, dtype=torch.uint8, device="cuda"), K)
    last = random_mx(g, 1, N, K)
    w.codes[-1], w.scales[-1] = last.codes[0], last.scales[0]
    T = (1 << 32) // (K // 2) + 40
    a = moe.MXTensor(torch.zeros((T, K // 2), dtype=torch.uint8, device="cuda"), torch.full((T, K // 32), 127, dtype=torch.uint8, device="cuda"), K)
    tail = random_mx(g, 7, K)
    a.codes[-7:], a.scales[-7:] = tail.codes, tail.scales
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[-1] = 7
    perm = (torch.arange(7, device="cuda") + T - 7).to(torch.int32)
    say("[mx product] large operands")
    y = moe.moe_mx_product(moe.make_mx_shape(7, K, N, E), a, w, offsets, perm=perm, out_dtype=F32)
    x, v = wide(tail), mx.values(last.codes[0], last.scales[0], K)
    near(y, x @ v.T, (K / 64 + 18) * 2.0 ** -23 * (x.abs() @ v.abs().T), "y")


@pytest.mark.parametrize("counts,K,widths", [
    ([1000], 4096, (15872, 7936)), ([1000], 1288, (40000, 20000)), ([1000], 896, (65536, 40968)), ([300, 5, 0, 513, 256, 64, 33, 1030], 4224, (6152, 3080)),
    ([191, 193, 512, 31, 224], 4104, (14344, 7176)), ([97] * 24, 7168, (6400, 3208)), ([2500, 0, 1, 0, 31, 33, 255, 257], 1408, (16000, 8008)), ([577, 640], 768, (65536, 51200))])
def test_large_tiles(counts, K, widths):
    """Wide enough for tiles of 256 x 256 to fill the chip more than once: products, then gate and up."""
    say(f"[mx product] {counts if len(counts) < 9 else len(counts)} {K} {widths}")
    check_product(make(counts, K, widths[0], spare=3))
    check_gate_up(make(counts, K, widths[1], tokens=77, k=2, pair=True))


def test_large_tiles_with_values_that_are_not_numbers_and_routings_that_do_not_fit():
    counts, N = [600, 130, 270], 15880
    say("[mx product] large tiles, not finite")
    s = make(counts, 4096, N, tokens=700, k=2, spare=3, pair=True, seed=9)
    s["perm"][:1000] = torch.arange(1000, device="cuda")
    run = lambda: (moe.moe_mx_product(s["shape"], s["a"], s["w"], s["offsets"], perm=s["perm"], k=2), moe.moe_mx_gate_up(s["shape"], s["a"], s["w"], s["u"], s["offsets"], perm=s["perm"], k=2))  # noqa: E731
    clean = run()
    s["a"].scales[200, 77] = 255               # rows 400 and 401
    s["w"].scales[2, N - 1, 3] = 255
    bad = torch.zeros((1003, N), dtype=torch.bool, device="cuda")
    bad[400:402] = True
    bad[730:1000, N - 1] = True
    bad[1000:] = True                          # (nobody's)
    for got, want in zip(run(), clean):
        assert torch.isnan(got[:1000][bad[:1000]]).all() and torch.equal(got[~bad], want[~bad])
    s["a"].scales[200, 77], s["w"].scales[2, N - 1, 3] = 127, 127
    clean = run()
    s["perm"][5], s["perm"][999], s["perm"][1001] = -9, 2 ** 31 - 1, 2 ** 31 - 1
    s["offsets"] = torch.tensor([-4, 600, 730, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    fine = [r for r in range(1000) if r not in (5, 999)]
    for got, want in zip(run(), clean):
        assert torch.equal(got[fine], want[fine])
