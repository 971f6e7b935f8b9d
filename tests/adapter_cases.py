"""Inputs, the plain form in 64 bits and error bounds of the projection with low-rank adapters."""
import random

import torch


def ids_of(pattern, T, n, seed=0):
    rng = random.Random(seed * 7919 + T)
    if pattern == "packed":     # a few requests, each a run of tokens
        ids, left = [], T
        while left > 0:
            m = min(left, rng.randint(1, max(1, T // 3)))
            ids += [rng.randrange(-1, n)] * m
            left -= m
    elif pattern == "scattered":
        ids = [rng.randrange(-1, n) for _ in range(T)]
    elif pattern == "one":
        ids = [n - 1] * T
    elif pattern == "none":
        ids = [-1] * T
    elif pattern == "each":
        ids = [t % n for t in range(T)]
    else:                       # "outside": ids that name no adapter
        ids = [rng.choice([0, n - 1, n, 2 ** 31 - 1, -7, -2 ** 31]) for _ in range(T)]
    return torch.tensor(ids, dtype=torch.int32, device="cuda")


def make(T, K, N, r, n, pattern, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(100 * seed + T)

    def normal(shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    s = {"ids": ids_of(pattern, T, n, seed), "scale": 0.5 + torch.rand(n, generator=g, device="cuda")}
    # the columns beside a row's own hold NaN: nothing may read them
    for name, width in (("x", K), ("dy", N)):
        wide = torch.full((T, width + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :width] = normal((T, width))
        s[name] = wide[:, :width]
    s["w"], s["a"], s["b"] = normal((K, N), K ** -0.5), normal((n, r, K), K ** -0.5), normal((n, r, N), 0.3)
    return s


def plain(s, scale=True):
    """Everything in 64 bits, token by adapter, and the sums of magnitudes that the bounds are made of."""
    x, dy, w, a, b = (s[k].double() for k in ("x", "dy", "w", "a", "b"))
    n, r, K = a.shape
    ids = s["ids"].long()
    sc = s["scale"].double() if scale else torch.ones(n, dtype=torch.float64, device="cuda")
    T, N = dy.shape
    z = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    v = {"y": x @ w, "dx": dy @ w.T, "h": z(T, r), "g": z(T, r), "da": z(n, r, K), "db": z(n, r, N)}
    m = {"y": x.abs() @ w.abs(), "dx": dy.abs() @ w.abs().T, "h": z(T, r), "g": z(T, r), "da": z(n, r, K), "db": z(n, r, N), "ylow": z(T, N), "dxlow": z(T, K)}
    for i in range(n):
        t = torch.nonzero(ids == i)[:, 0]
        if t.numel() == 0:
            continue
        h, g = sc[i] * (x[t] @ a[i].T), sc[i] * (dy[t] @ b[i].T)
        v["h"][t], v["g"][t] = h, g
        m["h"][t], m["g"][t] = sc[i] * (x[t].abs() @ a[i].abs().T), sc[i] * (dy[t].abs() @ b[i].abs().T)
        v["y"][t] += h @ b[i]
        v["dx"][t] += g @ a[i]
        m["ylow"][t], m["dxlow"][t] = h.abs() @ b[i].abs(), g.abs() @ a[i].abs()
        v["da"][i], v["db"][i] = g.T @ x[t], h.T @ dy[t]
        m["da"][i], m["db"][i] = g.abs().T @ x[t].abs(), h.abs().T @ dy[t].abs()
    return v, m


def low_error(s, m, name, of, factor):
    """What an error of h (or g) makes of the low-rank part: its sum over the ranks with the factor's magnitudes."""
    e = sums(m[name], of)
    out = torch.zeros((e.shape[0], factor.shape[2]), dtype=torch.float64, device="cuda")
    ids = s["ids"].long()
    for i in range(factor.shape[0]):
        t = torch.nonzero(ids == i)[:, 0]
        out[t] = e[t] @ factor[i].double().abs()
    return out


def sums(magnitude, terms):
    """Error of an fp32 sum: one rounding for every 16 products of a matrix instruction and for each of up to 64 parts, at worst
    half a step of 2^-23 of the magnitudes each; twice that, as the order inside an instruction is the hardware's."""
    return (terms / 16 + 64) * 2.0 ** -23 * magnitude


def bounds(s, v, m, out_f32):
    x, dy = s["x"], s["dy"]
    T, K = x.shape
    N = dy.shape[1]
    r = s["a"].shape[1]
    half = 2.0 ** -8   # of a bf16 value
    e = {"h": sums(m["h"], K)}
    # h as hi + lo: 2^-17 of its value, beside the error that h has; for an fp32 y it is kept whole
    e["y"] = sums(m["y"] + m["ylow"], K + 3 * r) + (0.0 if out_f32 else 2.0 ** -16) * m["ylow"] + low_error(s, m, "h", K, s["b"])
    e["dx"] = sums(m["dx"] + m["dxlow"], N + 2 * r) + 2.0 ** -16 * m["dxlow"] + low_error(s, m, "g", N, s["a"])
    if not out_f32:
        e["y"] = e["y"] + half * v["y"].abs()
    e["dx"] = e["dx"] + half * v["dx"].abs()
    ids = s["ids"].long()
    eh, eg = sums(m["h"], K), sums(m["g"], N)
    e["da"], e["db"] = sums(m["da"], T), sums(m["db"], T)
    for i in range(s["a"].shape[0]):
        t = torch.nonzero(ids == i)[:, 0]
        e["da"][i] += eg[t].T @ x[t].double().abs()
        e["db"][i] += eh[t].T @ dy[t].double().abs()
    return e


def check(got, want, err, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    bad = ~(off <= err + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), float((off / (err + 1e-30)).max()), torch.nonzero(bad)[:4].tolist())
