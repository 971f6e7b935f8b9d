"""Tokens to the rows of their experts and back, with the gradients, against the formulas in 64 bits."""
import random

import pytest
import torch

import paper_2604_19241_amd as moe
from helpers import say

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
KEEP = 7.0   # what rows that no slot names hold before and after


def table(T, k, rows, share, g):
    """[T,k] rows, every one at most once; the other slots name none."""
    row_of = torch.tensor([-1, -2 ** 31, 2 ** 31 - 1, rows], dtype=torch.int64)[torch.randint(0, 4, (T * k,), generator=g)]
    n = min(rows, int(round(share * T * k)))
    row_of[torch.randperm(T * k, generator=g)[:n]] = torch.randperm(rows, generator=g)[:n]
    return row_of.to(torch.int32).view(T, k).cuda()


def make(T, k, d, dtype, share=1.0, rows=None, pad=0, seed=0):
    g = torch.Generator().manual_seed(1000 * T + 10 * k + d + seed)
    rows = T * k if rows is None else rows
    s = {"T": T, "k": k, "d": d, "rows": rows, "dtype": dtype, "row_of": table(T, k, rows, share, g)}
    for name in ("x", "dy"):
        # the columns beside a row's own hold NaN: nothing may read them
        wide = torch.full((T, d + pad), float("nan"))
        wide[:, :d] = torch.randn((T, d), generator=g)
        s[name] = wide.to(dtype).cuda()[:, :d]
    s["w"] = torch.randn((T, k), generator=g).cuda()
    valid = (s["row_of"] >= 0) & (s["row_of"] < rows)
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[s["row_of"][valid].long()] = True
    s["named"], s["valid"] = named, valid
    for name in ("o", "dxs"):
        v = torch.randn((rows, d), generator=g).cuda()
        v[~named] = float("nan")   # nor the rows that no slot names
        s[name] = v.to(dtype)
    s["shape"] = moe.make_dispatch_shape(T, k, d, rows)
    return s


def gathered(s, name):
    v = s[name].double()[torch.where(s["valid"], s["row_of"], 0).long()] if s["rows"] else torch.zeros((s["T"], s["k"], s["d"]), dtype=torch.float64, device="cuda")
    return torch.where(s["valid"][:, :, None], v, 0.0)


def half(s, want):
    """Half a step of the result's type, relative to the value."""
    return (2.0 ** -8 if s["dtype"] is BF else 2.0 ** -24) * want.abs()


def near(got, want, err, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    assert (off <= err + 1e-38).all(), (what, float((off - err).max()))


def check(s):
    T, k, d, rows, shape, row_of, w = (s[n] for n in ("T", "k", "d", "rows", "shape", "row_of", "w"))
    flat, valid = row_of.view(-1).long(), s["valid"].view(-1)

    def kept():
        return torch.full((rows, d), KEEP, dtype=s["dtype"], device="cuda")

    xs = moe.moe_dispatch_forward(shape, s["x"], row_of, out=kept())
    want = kept()
    want[flat[valid]] = s["x"].repeat_interleave(k, 0)[valid]
    assert torch.equal(xs, want)

    dx = moe.moe_dispatch_backward(shape, s["dxs"], row_of)
    v = gathered(s, "dxs")
    # k - 1 fp32 additions, each off by half a step of at most the sum of the magnitudes, and the result's rounding
    near(dx, v.sum(1), k * 2.0 ** -24 * v.abs().sum(1) + half(s, v.sum(1)), "dx")

    for weights in (w, None):
        o, ww = gathered(s, "o"), (w if weights is not None else torch.ones_like(w)).double()
        terms = o * ww[:, :, None]
        y = moe.moe_combine_forward(shape, s["o"], row_of, weights)
        near(y, terms.sum(1), k * 2.0 ** -24 * terms.abs().sum(1) + half(s, terms.sum(1)), "y")
        got = moe.moe_combine_backward(shape, s["dy"], s["o"], row_of, weights, out={"do": kept()})
        do = kept().double()
        do[flat[valid]] = (ww[:, :, None] * s["dy"].double()[:, None]).view(T * k, d)[valid]
        # one product in fp32, and the rounding
        err = 2.0 ** -24 * do.abs() + half(s, do)
        err[~s["named"]] = 0.0
        near(got["do"], do, err, "do")
        dots = o * s["dy"].double()[:, None]
        # a lane's chain of products, six steps over the lanes and three over the waves
        near(got["dw"], dots.sum(2), (d / 256 + 8 + 9) * 2.0 ** -24 * dots.abs().sum(2), "dw")
        again = moe.moe_combine_backward(shape, s["dy"], None, row_of, weights, want_dw=False, out={"do": kept()})
        assert again["dw"] is None and torch.equal(again["do"], got["do"])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,k,d,share,pad", [(1, 1, 8, 1.0, 0), (1, 8, 2048, 1.0, 0), (1, 16, 7168, 0.5, 8), (3, 2, 72, 0.5, 8), (64, 3, 512, 1.0, 0), (65, 9, 520, 0.7, 64),
                                             (700, 8, 2304, 0.3, 0), (257, 4, 1032, 1.0, 8), (33, 16, 264, 1.0, 0), (500, 1, 16, 0.1, 0), (40, 5, 104, 0.0, 0)])
def test_every_direction(T, k, d, share, pad, dtype):
    say(f"[move] {T} {k} {d} {share} {pad} {dtype}")
    check(make(T, k, d, dtype, share, pad=pad))


@pytest.mark.parametrize("rows", [0, 1, 100, 5000])
def test_buffers_of_other_sizes_than_the_slots(rows):
    say(f"[move] {rows} rows")
    check(make(60, 4, 136, BF, 0.8, rows=rows))


def test_no_tokens():
    shape = moe.make_dispatch_shape(0, 4, 64, 10)
    row_of = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    buf = torch.full((10, 64), KEEP, dtype=BF, device="cuda")
    none = torch.empty((0, 64), dtype=BF, device="cuda")
    assert (moe.moe_dispatch_forward(shape, none, row_of, out=buf) == KEEP).all()
    assert moe.moe_combine_forward(shape, buf, row_of).shape == (0, 64)
    got = moe.moe_combine_backward(shape, none, buf.clone(), row_of, out={"do": buf})
    assert (got["do"] == KEEP).all() and got["dw"].shape == (0, 4)


def test_the_gradients_are_differences():
    """Both sums are linear in each argument, so a central difference is the gradient: here with steps that fp32 keeps exactly."""
    s = make(3, 2, 8, F32, 0.9, seed=3)
    o = torch.where(s["named"][:, None], s["o"], 0.0)
    o, w, dy, x = ((v * 64).round() / 64 for v in (o, s["w"], s["dy"], s["x"]))
    shape, row_of = s["shape"], s["row_of"]

    def loss(o, w):
        return float((moe.moe_combine_forward(shape, o, row_of, w).double() * dy.double()).sum())

    got = moe.moe_combine_backward(shape, dy, o, row_of, w, out={"do": torch.zeros_like(o)})
    for v, grad in ((o, got["do"]), (w, got["dw"])):
        for i in range(v.numel()):
            up, down = v.clone(), v.clone()
            up.view(-1)[i] += 1
            down.view(-1)[i] -= 1
            pair = [(a, w) if v is o else (o, a) for a in (up, down)]
            assert abs((loss(*pair[0]) - loss(*pair[1])) / 2 - float(grad.view(-1)[i])) <= 1e-4   # (sums of up to 48 products below 16 in fp32)
    dxs = torch.where(s["named"][:, None], s["dxs"], 0.0)
    dx = moe.moe_dispatch_backward(shape, dxs, row_of)
    for i in range(x.numel()):
        sides = []
        for step in (1, -1):
            v = x.clone()
            v.view(-1)[i] += step
            sides.append(float((moe.moe_dispatch_forward(shape, v, row_of, out=torch.zeros_like(dxs)).double() * dxs.double()).sum()))
        assert abs((sides[0] - sides[1]) / 2 - float(dx.view(-1)[i])) <= 1e-4


def test_values_that_are_not_finite_stay_with_their_token():
    s = make(50, 4, 72, BF, 0.9)
    t, j = torch.nonzero(s["valid"])[5].tolist()
    o = torch.where(s["named"][:, None], s["o"], 0.0)
    clean = moe.moe_combine_forward(s["shape"], o, s["row_of"], s["w"])
    bad = o.clone()
    bad[s["row_of"][t, j].long(), 3] = float("inf")
    y = moe.moe_combine_forward(s["shape"], bad, s["row_of"], s["w"])
    assert torch.isinf(y[t, 3]) and not torch.isfinite(y[t, 3])
    y[t, 3] = clean[t, 3]
    assert torch.equal(y, clean)
    w = s["w"].clone()
    w[t, j] = 0.0
    assert torch.isnan(moe.moe_combine_forward(s["shape"], bad, s["row_of"], w)[t, 3])   # 0 times infinity, as in the formula


@pytest.mark.parametrize("dtype", [BF, F32])
def test_offsets_beyond_32_bits(dtype):
    rows, d = (1 << 32) // 2304 + 1000, 2304
    shape = moe.make_dispatch_shape(4, 2, d, rows)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((4, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    row_of = torch.tensor([[rows - 1, 0], [-1, rows - 7], [rows, 5], [rows - 3, rows - 2]], dtype=torch.int32, device="cuda")
    ok = (row_of >= 0) & (row_of < rows)
    w = torch.randn((4, 2), generator=g, device="cuda")
    buf = torch.zeros((rows, d), dtype=dtype, device="cuda")
    say("[move] large buffer")
    moe.moe_dispatch_forward(shape, x, row_of, out=buf)
    token = torch.arange(4, device="cuda")[:, None].expand(4, 2)[ok]
    at = row_of[ok].long()
    assert torch.equal(buf[at], x[token])
    n = ok.sum(1, keepdim=True)
    assert torch.equal(moe.moe_dispatch_backward(shape, buf, row_of), (x.float() * n).to(dtype))   # (x + x is exact)
    dw = moe.moe_combine_backward(shape, dy, buf, row_of, w, out={"do": torch.empty_like(buf)})["dw"]
    want = torch.where(ok, (dy.double() * x.double()).sum(1, keepdim=True), 0.0)
    assert ((dw - want).abs() <= 26 * 2.0 ** -24 * (dy.double() * x.double()).abs().sum(1, keepdim=True)).all()


def test_routing_and_global_map_as_tables():
    """moe_route's inv_perm of a share of the experts, and the send buffers of one rank of two."""
    T, E, k, d = 300, 16, 4, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    logits = torch.randn((T, E), generator=g, device="cuda")
    x = torch.randn((T, d), generator=g, device="cuda").to(BF)
    r = moe.moe_route(moe.make_shape(T, d, E, k, 64, 4, 8), logits)
    A = int(r.offsets[-1])
    xs = moe.moe_dispatch_forward(moe.make_dispatch_shape(T, k, d), x, r.inv_perm)
    assert torch.equal(xs[:A], x[r.perm[:A].long() // k])
    shape = moe.make_shape(T, d, E, k, 64)
    r = moe.moe_route(shape, logits)
    m = moe.moe_global_map(shape, 2, 0, r, torch.stack([r.counts, torch.zeros_like(r.counts)]))
    mine = torch.where(m.dst_rank == 1, m.dst_row, -1)   # what goes to the other rank
    n = int(r.counts[E // 2:].sum())
    sent = moe.moe_dispatch_forward(moe.make_dispatch_shape(T, k, d, n), x, mine)
    assert torch.equal(sent, x[r.perm[int(r.offsets[E // 2]):].long() // k])


def test_streams_and_graphs():
    s = make(90, 4, 264, BF, 0.8)
    o, dxs = (torch.where(s["named"][:, None], s[n], 0.0) for n in ("o", "dxs"))
    x, dy, w, row_of = s["x"].clone(), s["dy"].clone(), s["w"].clone(), s["row_of"].clone()
    buf = [torch.zeros_like(o) for _ in range(2)]

    def run():
        xs = moe.moe_dispatch_forward(s["shape"], x, row_of, out=buf[0])
        dx = moe.moe_dispatch_backward(s["shape"], dxs, row_of)
        y = moe.moe_combine_forward(s["shape"], o, row_of, w)
        g = moe.moe_combine_backward(s["shape"], dy, o, row_of, w, out={"do": buf[1]})
        return [xs, dx, y, g["do"], g["dw"]]

    want = [v.clone() for v in run()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        x.zero_(), dy.zero_()
        torch.cuda._sleep(40_000_000)   # the inputs are not there before that is over
        x.copy_(s["x"]), dy.copy_(s["dy"])
        got = [v.clone() for v in run()]
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for step in range(4):
        x.copy_(s["x"] * (step + 1))
        dy.copy_(s["dy"] * (step + 1))
        graph.replay()
        got = [v.clone() for v in out]
        torch.cuda.synchronize()
        want = run()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), step
