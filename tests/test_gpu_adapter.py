"""The shared projection with low-rank adapters, forward and backward, against the plain form in 64 bits."""
import pytest
import torch

import adapter_cases as ac
import paper_2604_19241_amd as moe
from helpers import say

pytestmark = pytest.mark.gpu


def run(s, r, n, out_dtype=torch.bfloat16, backward=True, scale=True):
    T, K = s["x"].shape
    N = s["dy"].shape[1]
    shape = moe.make_adapter_shape(T, K, N, r, n)
    plan = moe.moe_adapter_plan(shape, s["ids"])
    h = torch.full((T, r), float("nan"), device="cuda")
    sc = s["scale"] if scale else None
    out = {"y": moe.moe_adapter_forward(shape, s["x"], s["w"], s["a"], s["b"], plan, scale=sc, out_dtype=out_dtype, h=h), "h": h}
    if backward:
        out |= moe.moe_adapter_backward(shape, s["dy"], s["x"], s["w"], s["a"], s["b"], plan, h, scale=sc)
    return out


CASES = [  # T, K, N, rank, adapters, ids, pad, out
    (1, 64, 64, 8, 1, "one", 0, "bf16"), (1, 2048, 512, 16, 8, "one", 0, "bf16"), (1, 8, 8, 8, 3, "none", 8, "f32"),
    (2, 72, 24, 8, 5, "each", 0, "bf16"), (31, 200, 136, 24, 4, "packed", 8, "bf16"), (32, 520, 1032, 40, 3, "scattered", 0, "f32"),
    (33, 1000, 88, 16, 64, "each", 64, "bf16"), (64, 4096, 40, 128, 2, "scattered", 0, "bf16"), (65, 328, 640, 72, 7, "outside", 0, "bf16"),
    (200, 136, 2056, 8, 256, "each", 0, "bf16"), (256, 448, 264, 128, 1, "one", 0, "f32"), (256, 512, 1024, 8, 2, "packed", 0, "bf16"),
    (257, 64, 64, 8, 1, "one", 0, "bf16"), (257, 8, 16, 8, 300, "each", 0, "f32"), (300, 328, 200, 24, 5, "outside", 8, "bf16"),
    (512, 1160, 264, 96, 2, "one", 0, "bf16"), (500, 72, 2056, 128, 9, "scattered", 0, "bf16"), (301, 2056, 136, 128, 2, "each", 0, "bf16"),
    (500, 72, 3000, 128, 20, "scattered", 0, "f32"), (500, 2200, 72, 128, 3, "scattered", 0, "bf16"), (64, 16400, 40, 128, 2, "scattered", 0, "bf16"), (500, 72, 2056, 16, 9, "scattered", 0, "bf16"),
    # more tokens: sorted by adapter
    (513, 64, 64, 8, 1, "one", 0, "bf16"), (513, 8, 16, 8, 600, "each", 0, "f32"), (600, 328, 200, 24, 5, "outside", 8, "bf16"),
    (1011, 136, 72, 16, 256, "scattered", 0, "bf16"), (640, 1000, 520, 64, 3, "packed", 64, "f32"), (1021, 264, 712, 128, 2, "scattered", 0, "bf16"),
    (1000, 200, 104, 40, 1024, "scattered", 0, "bf16"), (2049, 512, 128, 8, 4, "packed", 0, "f32"), (777, 72, 640, 96, 6, "none", 0, "bf16"),
    (900, 264, 392, 16, 300, "each", 0, "bf16"), (1500, 2056, 136, 64, 500, "scattered", 0, "f32"), (2000, 136, 3000, 8, 30, "packed", 0, "bf16"),
    # tiles of 128 and of 256 rows, in each direction
    (4100, 136, 1032, 16, 9, "packed", 0, "bf16"), (4100, 1032, 72, 16, 300, "scattered", 0, "bf16"), (8200, 72, 1544, 24, 6, "scattered", 8, "bf16"),
    (8200, 1544, 136, 64, 5, "packed", 0, "f32"), (16500, 584, 1032, 8, 40, "scattered", 0, "f32"), (16500, 1032, 584, 128, 3, "packed", 0, "bf16"),
    (16500, 136, 72, 48, 7, "scattered", 0, "bf16"),
    # an adapter's rows in several parts
    (4099, 264, 136, 16, 1, "one", 0, "bf16"), (3000, 72, 200, 72, 2, "scattered", 0, "bf16"), (5000, 392, 72, 8, 3, "none", 0, "f32"),
    # parts of a long reduction in both directions, few tokens and sorted ones
    (600, 1544, 1600, 16, 7, "scattered", 0, "bf16"), (2600, 3000, 24, 8, 12, "packed", 8, "bf16"), (1100, 24, 2056, 128, 3, "scattered", 0, "f32"),
    (900, 1552, 1608, 24, 300, "each", 0, "f32"), (3000, 1600, 520, 40, 2, "one", 0, "bf16"),
    (40, 7000, 4104, 16, 3, "scattered", 0, "bf16"), (400, 5000, 264, 24, 2, "packed", 8, "f32"),
    # a batch on few of many adapters: rows in parts, by adapter or by those with many rows
    (12337, 72, 24, 16, 193, "packed", 0, "bf16"), (2206, 616, 2320, 64, 189, "packed", 0, "bf16"), (5000, 136, 72, 8, 300, "one", 8, "f32"), (6000, 264, 136, 24, 20, "one", 0, "bf16"),
    (8200, 72, 136, 16, 12, "packed", 0, "bf16"), (3000, 72, 200, 72, 40, "none", 0, "bf16"), (3000, 72, 200, 72, 9, "none", 0, "bf16"), (9000, 24, 8, 128, 130, "outside", 0, "bf16"),
    (4000, 136, 264, 16, 8, "scattered", 0, "bf16"), (1100, 2056, 3000, 8, 16, "packed", 0, "bf16"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_the_plain_form(case):
    T, K, N, r, n, pattern, pad, out = case
    say(f"[adapter] {case}")
    s = ac.make(T, K, N, r, n, pattern, pad)
    got = run(s, r, n, torch.float32 if out == "f32" else torch.bfloat16)
    torch.cuda.synchronize()
    v, m = ac.plain(s)
    e = ac.bounds(s, v, m, out == "f32")
    for key in ("h", "y", "dx", "da", "db"):
        ac.check(got[key], v[key], e[key], (case, key))


def test_without_scale_and_without_the_stash():
    for T in (40, 700):
        s = ac.make(T, 136, 200, 16, 3, "packed")
        got = run(s, 16, 3, scale=False)
        v, m = ac.plain(s, scale=False)
        e = ac.bounds(s, v, m, False)
        for key in ("h", "y", "dx", "da", "db"):
            ac.check(got[key], v[key], e[key], (T, key))
        shape = moe.make_adapter_shape(T, 136, 200, 16, 3)
        assert torch.equal(moe.moe_adapter_forward(shape, s["x"], s["w"], s["a"], s["b"], moe.moe_adapter_plan(shape, s["ids"])), got["y"])


def test_up_to_512_tokens_with_and_without_a_plan():
    T, K, N, r, n = 420, 4616, 4616, 16, 5
    s = ac.make(T, K, N, r, n, "scattered")
    shape = moe.make_adapter_shape(T, K, N, r, n)
    v, m = ac.plain(s)
    e = ac.bounds(s, v, m, False)
    plan = moe.moe_adapter_plan(shape, s["ids"])
    assert plan.table is not None
    for p in (plan, moe.AdapterPlan(s["ids"], None)):
        h = torch.empty((T, r), device="cuda")
        got = {"y": moe.moe_adapter_forward(shape, s["x"], s["w"], s["a"], s["b"], p, scale=s["scale"], h=h), "h": h}
        got |= moe.moe_adapter_backward(shape, s["dy"], s["x"], s["w"], s["a"], s["b"], p, h, scale=s["scale"])
        for key in ("h", "y", "dx", "da", "db"):
            ac.check(got[key], v[key], e[key], (p.table is None, key))


def test_a_plan_serves_other_widths():
    T, r, n = 700, 16, 5
    one, two = ac.make(T, 136, 264, r, n, "scattered"), ac.make(T, 520, 72, 40, n, "scattered")
    plan = moe.moe_adapter_plan(moe.make_adapter_shape(T, 136, 264, r, n), one["ids"])
    two["ids"] = one["ids"]
    with pytest.raises(AssertionError):   # but no other number of adapters
        six = ac.make(T, 520, 72, 40, 6, "scattered")
        moe.moe_adapter_forward(moe.make_adapter_shape(T, 520, 72, 40, 6), six["x"], six["w"], six["a"], six["b"], plan)
    y = moe.moe_adapter_forward(moe.make_adapter_shape(T, 520, 72, 40, n), two["x"], two["w"], two["a"], two["b"], plan, scale=two["scale"])
    assert torch.equal(y, run(two, 40, n, backward=False)["y"])


def test_no_tokens():
    s = ac.make(0, 64, 128, 8, 3, "one")
    got = run(s, 8, 3)
    assert got["y"].shape == (0, 128) and got["dx"].shape == (0, 64)
    assert not got["da"].any() and not got["db"].any() and got["da"].shape == (3, 8, 64)


@pytest.mark.parametrize("T,K,N", [(48, 264, 392), (512, 64, 512), (700, 264, 392), (4200, 72, 1032), (4200, 1032, 72), (8300, 72, 1544), (8300, 1544, 72)])
def test_an_adapter_that_is_not_finite_stays_with_its_tokens(T, K, N):
    """Rows, and factors' gradients, of every other adapter are the same bits as with a finite one in its place."""
    r, n = 16, 4
    s = ac.make(T, K, N, r, n, "scattered")
    clean = run(s, r, n)
    for name, value in (("b", float("nan")), ("b", float("inf")), ("a", float("inf")), ("a", float("nan"))):
        say(f"[adapter] {T} {K} {N}: {name} holds {value}")
        bad = dict(s)
        bad[name] = s[name].clone()
        bad[name][2, 3, 5] = value
        got = run(bad, r, n)
        others = s["ids"] != 2
        for key in ("y", "h"):
            assert torch.isfinite(got[key][others].float()).all()
        # (a tile that is added up again without its low-rank part rounds another fp32 sum)
        v, m = ac.plain(s)
        e = ac.bounds(s, v, m, False)
        for key in ("y", "dx"):
            ac.check(got[key][others], v[key][others], e[key][others], (T, name, value, key))
            assert not torch.isfinite(got["y"][~others].float()).all() or not torch.isfinite(got["dx"][~others].float()).all()
        assert torch.equal(got["h"][others], clean["h"][others])
        for i in (0, 1, 3):
            assert torch.equal(got["da"][i], clean["da"][i]) and torch.equal(got["db"][i], clean["db"][i])


@pytest.mark.parametrize("T", [37, 900, 8300])
def test_the_same_bits_every_time(T):
    K, N, r, n = 264, 1544, 24, 5
    s = ac.make(T, K, N, r, n, "packed")
    one, two = run(s, r, n), run(s, r, n)
    assert all(torch.equal(one[key], two[key]) for key in one)


def test_gradients_are_the_differences_of_the_forward_pass():
    """y is linear in each factor, so that a difference over any step is the slope: of sum(dy y) by single elements."""
    for T in (20, 600):
        K, N, r, n = 64, 72, 8, 3
        s = ac.make(T, K, N, r, n, "packed", seed=3)
        got = run(s, r, n, torch.float32)
        v, m = ac.plain(s)
        e = ac.bounds(s, v, m, True)

        def loss(part):
            return float((run(part, r, n, torch.float32, backward=False)["y"].double() * s["dy"].double()).sum())

        err = float((e["y"] * s["dy"].double().abs()).sum())
        for name, grad in (("a", "da"), ("b", "db")):
            for at in ((0, 0, 0), (2, 7, 63), (1, 3, 17)):
                step = 4.0
                up, down = dict(s), dict(s)
                up[name], down[name] = s[name].clone(), s[name].clone()
                up[name][at] = step
                down[name][at] = -step
                slope = (loss(up) - loss(down)) / (2 * step)
                # (the perturbed forward passes are off by what theirs is: a few times the unperturbed bound)
                assert abs(slope - float(got[grad][at])) <= 8 * err / step + float(e[grad][at]), (T, name, at)


def test_in_a_graph_and_behind_other_work_of_the_stream():
    for T, N in ((48, 392), (700, 392), (4200, 1032)):
        K, r, n = 264, 16, 4
        s = ac.make(T, K, N, r, n, "scattered")
        shape = moe.make_adapter_shape(T, K, N, r, n)
        want = run(s, r, n)
        torch.cuda.synchronize()
        buf = {k: torch.zeros_like(v) for k, v in s.items()}
        ws = torch.empty(moe.moe_adapter_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
        h = torch.empty((T, r), device="cuda")

        def step():
            plan = moe.moe_adapter_plan(shape, buf["ids"])
            y = moe.moe_adapter_forward(shape, buf["x"], buf["w"], buf["a"], buf["b"], plan, scale=buf["scale"], h=h, ws=ws)
            return {"y": y} | moe.moe_adapter_backward(shape, buf["dy"], buf["x"], buf["w"], buf["a"], buf["b"], plan, h, scale=buf["scale"], ws=ws)

        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)
            for k, v in s.items():
                buf[k].copy_(v)
            eager = step()
        stream.synchronize()
        assert all(torch.equal(eager[k], want[k]) for k in eager), T
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        for turn in range(3):
            for t in out.values():
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], want[k]) for k in out), (T, turn)
            assert all(torch.equal(v, want[k]) for k, v in step().items()), (T, turn)


def test_other_tensors_are_refused():
    T, K, N, r, n = 40, 64, 72, 8, 3
    s = ac.make(T, K, N, r, n, "scattered", 8)
    shape = moe.make_adapter_shape(T, K, N, r, n)
    plan = moe.moe_adapter_plan(shape, s["ids"])
    h = torch.zeros((T, r), device="cuda")
    forward = {"x": s["x"], "w": s["w"], "a": s["a"], "b": s["b"], "scale": s["scale"], "h": h}
    backward = forward | {"dy": s["dy"]}

    def call(back, kw):
        kw, args = dict(kw), [shape]
        for name in ("dy", "x", "w", "a", "b") if back else ("x", "w", "a", "b"):
            args.append(kw.pop(name))
        (moe.moe_adapter_backward if back else moe.moe_adapter_forward)(*args, plan, **kw)

    call(False, forward)
    call(True, backward)
    for back, good in ((False, forward), (True, backward)):
        for name, t in good.items():
            wrong = [t.cpu(), t.double(), t[..., :-1], t[None]]
            if t.dim() > 1:
                wrong.append(t.transpose(-1, -2).contiguous().transpose(-1, -2))   # right sizes, the other order
            for bad in wrong:
                with pytest.raises(AssertionError):
                    call(back, good | {name: bad})
    with pytest.raises(AssertionError):
        call(False, forward | {"y": torch.empty((T, N), device="cuda")})           # fp32 where bf16 is asked for
    with pytest.raises(AssertionError):
        call(False, forward | {"ws": torch.empty(1 << 20, device="cuda")})
    with pytest.raises(RuntimeError):
        call(False, forward | {"ws": torch.empty(0, dtype=torch.uint8, device="cuda")})   # too small
    for bad in (s["ids"].long(), s["ids"][:-1], s["ids"].cpu()):
        with pytest.raises(AssertionError):
            moe.moe_adapter_plan(shape, bad)


@pytest.mark.parametrize("T,K,N,r,n", [(5, 64, 72, 8, 4), (48, 264, 392, 16, 4), (300, 136, 264, 16, 100), (512, 64, 512, 16, 4), (700, 264, 392, 16, 4), (900, 1552, 1608, 24, 300), (1011, 136, 72, 16, 256),
                                       (4200, 72, 1032, 16, 4), (4200, 1032, 72, 64, 5), (8300, 1544, 136, 16, 4), (3000, 72, 200, 72, 2), (16500, 584, 264, 128, 3)])
def test_tokens_that_are_not_finite_stay_by_themselves(T, K, N, r, n):
    """Other tokens' rows, and the gradients of adapters that have none of these tokens."""
    s = ac.make(T, K, N, r, n, "scattered")
    clean = run(s, r, n)
    v, m = ac.plain(s)
    e = ac.bounds(s, v, m, False)
    ids = s["ids"]
    for where in (ids == 1, (ids == -1)):
        for name, value in (("x", float("nan")), ("x", float("inf")), ("dy", float("-inf")), ("dy", float("nan"))):
            say(f"[adapter] {T} {K} {N}: {name} holds {value}")
            bad = dict(s)
            bad[name] = s[name].clone()
            bad[name][where, 3:9] = value
            got = run(bad, r, n)
            for key in ("y", "dx"):
                ac.check(got[key][~where], v[key][~where], e[key][~where], (T, name, value, key))
            assert torch.equal(got["h"][~where], clean["h"][~where])
            for i in range(n):
                if not (where & (ids == i)).any():
                    assert torch.equal(got["da"][i], clean["da"][i]) and torch.equal(got["db"][i], clean["db"][i]), (name, value, i)


def test_offsets_beyond_32_bits():
    """Rows that lie far apart, and results of more than 2^32 bytes."""
    g = torch.Generator(device="cuda").manual_seed(5)
    for T, K, N, apart in ((600, 64, 72, 1 << 22), (40, 64, 72, 1 << 26), (34000, 64, 65536, 0)):
        say(f"[adapter] {T} {K} {N}, rows {apart} apart")
        r, n = 16, 3
        s = ac.make(min(T, 2), K, 8, r, n, "one")   # (w and b below)
        wide = torch.empty((T, max(apart, K)), dtype=torch.bfloat16, device="cuda")
        wide[:, :K] = torch.randn((T, K), generator=g, device="cuda").to(torch.bfloat16)
        s |= {"x": wide[:, :K], "ids": ac.ids_of("scattered", T, n), "w": (torch.randn((K, N), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16),
              "b": (torch.randn((n, r, N), generator=g, device="cuda") * 0.3).to(torch.bfloat16)}
        dy = torch.empty((T, max(apart, N)), dtype=torch.bfloat16, device="cuda")
        for i in range(0, T, 2000):
            dy[i:i + 2000, :N] = torch.randn((min(2000, T - i), N), generator=g, device="cuda").to(torch.bfloat16)
        s["dy"] = dy[:, :N]
        got = run(s, r, n)
        # rows of the results by themselves, and a few columns of the gradient that every row of dy is part of
        at = torch.tensor(sorted({0, 1, T // 2, T - 2, T - 1} | set(range(0, T, max(1, T // 40)))), device="cuda")
        few = {k: v[at].contiguous() if k in ("x", "dy", "ids") else v for k, v in s.items()}
        v, m = ac.plain(few)
        e = ac.bounds(few, v, m, False)
        for key in ("h", "y", "dx"):
            ac.check(got[key][at], v[key], e[key], (T, apart, key))
        cols = torch.tensor([0, 1, N // 2, N - 1], device="cuda")
        part = {"x": s["x"], "ids": s["ids"], "scale": s["scale"], "a": s["a"], "w": s["w"][:, cols], "b": s["b"][:, :, cols], "dy": s["dy"][:, cols]}
        v, m = ac.plain(part)
        e = ac.bounds(part, v, m, False)
        ac.check(got["db"][:, :, cols], v["db"], e["db"], (T, apart, "db"))
        del got, s, wide, dy


@pytest.mark.parametrize("T", [257, 400, 512])
def test_a_plan_of_257_to_512_tokens_serves_all_widths(T):
    """Narrow shapes do not sort so few tokens and wide ones do: the results of either are the same bits whichever the plan was made with, or without one."""
    import ctypes
    r, n = 16, 5
    sizes = {"narrow": (512, 136), "wide": (5800, 5800)}
    s = {k: ac.make(T, K, N, r, n, "scattered") for k, (K, N) in sizes.items()}
    s["wide"]["ids"] = s["narrow"]["ids"]
    ids = s["narrow"]["ids"]
    shape = {k: moe.make_adapter_shape(T, K, N, r, n) for k, (K, N) in sizes.items()}
    plans = {k: moe.moe_adapter_plan(shape[k], ids) for k in sizes}
    assert plans["narrow"].table is None and plans["wide"].table is not None
    # a caller of the C interface with one buffer for its widest layer, filled by its first
    table = torch.full_like(plans["wide"].table, -1)
    lib = moe.load_library()
    assert lib.moe_adapter_plan(ctypes.byref(shape["narrow"]), ids.data_ptr(), table.data_ptr(), 4 * table.numel(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    blocks = int(plans["wide"].table[0])
    assert int(table[0]) == blocks and torch.equal(table[16:16 + 2 * blocks], plans["wide"].table[16:16 + 2 * blocks])
    plans |= {"filled": moe.AdapterPlan(ids, table, n), "none": moe.AdapterPlan(ids, None)}
    for k in sizes:
        v, m = ac.plain(s[k])
        e = ac.bounds(s[k], v, m, False)
        want = None
        for name, plan in plans.items():
            h = torch.empty((T, r), device="cuda")
            got = {"y": moe.moe_adapter_forward(shape[k], s[k]["x"], s[k]["w"], s[k]["a"], s[k]["b"], plan, scale=s[k]["scale"], h=h), "h": h}
            got |= moe.moe_adapter_backward(shape[k], s[k]["dy"], s[k]["x"], s[k]["w"], s[k]["a"], s[k]["b"], plan, h, scale=s[k]["scale"])
            for key in got:
                ac.check(got[key], v[key], e[key], (T, k, name, key))
            want = want or got
            assert all(torch.equal(got[key], want[key]) for key in got), (T, k, name)


@pytest.mark.parametrize("T,N", [(40, 72), (300, 72), (700, 72), (420, 4616)])
def test_a_table_that_is_not_the_batch_s_own_is_refused(T, N):
    K, r, n = (64 if N == 72 else 4616), 8, 3
    s = ac.make(T, K, N, r, n, "scattered")
    shape = moe.make_adapter_shape(T, K, N, r, n)
    plan = moe.moe_adapter_plan(shape, s["ids"])
    h = torch.zeros((T, r), device="cuda")
    table = plan.table
    if table is None and T > 256:   # that of a wider layer
        table = moe.moe_adapter_plan(moe.make_adapter_shape(T, 1 << 16, 1 << 16, r, n), s["ids"]).table

    def both(t):
        p = moe.AdapterPlan(s["ids"], t, n)
        return (lambda: moe.moe_adapter_forward(shape, s["x"], s["w"], s["a"], s["b"], p, h=h),
                lambda: moe.moe_adapter_backward(shape, s["dy"], s["x"], s["w"], s["a"], s["b"], p, h))

    wrong = [moe.moe_adapter_plan(moe.make_adapter_shape(t, K, N, r, n), ac.ids_of("scattered", t, n)).table for t in (600, T + 513)]   # ids were replaced since
    if table is not None:
        for call in both(table):
            call()
        wrong += [table[:-1], torch.cat([table, table]), torch.cat([table, table[:1]]), torch.stack([table, table], 1)[:, 0], table.long(), table.float(), table.cpu(), table[:0]]
    for t in wrong:
        for call in both(t):
            with pytest.raises(AssertionError):
                call()
    torch.cuda.synchronize()


def test_memory_that_is_not_there_raises_as_torch_does():
    T, K, N, r, n = 1 << 20, 8, 16384, 8, 2   # a result of 32 GiB
    s = ac.make(4, K, N, r, n, "one")
    x, ids = torch.zeros((T, K), dtype=torch.bfloat16, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    shape = moe.make_adapter_shape(T, K, N, r, n)
    plan = moe.moe_adapter_plan(shape, ids)
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(0.05)   # torch's allocator refuses more by itself
    try:
        with pytest.raises(torch.OutOfMemoryError):
            torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
        with pytest.raises(torch.OutOfMemoryError):
            moe.moe_adapter_forward(shape, x, s["w"], s["a"], s["b"], plan)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
