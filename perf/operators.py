"""The operators beside the routed experts, and the workloads that their speed is followed on.

A case is one pass as a user's program makes it:

  project  the shared projection of T packed tokens of `requests` requests, each with one of `adapters` low-rank
           adapters (`bare` of them with none): y = x W + scale (x A^T) B, in serving, where nothing is kept;
  tune     the same in a training step, and the gradients of x and of every adapter's two factors (W is frozen);
  balance  a router's balance loss and z loss over T tokens of `seqs` packed sequences with the count of every
           expert, and the gradient of the logits, that of the selected gates included.

K and N are the projection's inner and outer widths, E experts of which k are selected.  `own` selects the
framework's kernels; otherwise the same is computed by plain torch operations in 32 bits.
"""
import math
import random

import torch

own = False

BALANCE_COEF, Z_COEF = 0.01, 0.001


def _projection(kind, T, K, N, rank, adapters, requests, bare=0, out="bf16", pad=0):
    return {"kind": kind, "T": T, "K": K, "N": N, "rank": rank, "adapters": adapters, "requests": requests,
            "bare": bare, "out": out, "pad": pad}


def _balance(T, E, k, seqs=1, padding=0.0, gates=True, out="f32"):
    return {"kind": "balance", "T": T, "E": E, "k": k, "seqs": seqs, "padding": padding, "gates": gates, "out": out}


def listed():
    cases = {
        # one sequence generating, one adapter of eight: latency and the stream of W
        "project-1": _projection("project", 1, 2048, 2048, 16, 8, 1),
        # a generation step of many requests, most with an adapter of their own, two with none
        "project-37": _projection("project", 37, 7168, 2048, 16, 64, 37, bare=2),
        # a large generation step, more adapters than rows of a tile, in both factors as many bytes as W
        "project-256": _projection("project", 256, 2048, 4096, 8, 256, 256),
        # a few prompts of odd lengths through the up-projection of a shared expert; x is a part of a wider buffer
        "project-1021": _projection("project", 1021, 2048, 2816, 32, 16, 5, bare=1, pad=64),
        # a long batch of prompts, wide in, down to the inner width
        "project-8192": _projection("project", 8192, 7168, 2048, 16, 16, 24, bare=3),
        # a router's logits, in 32 bits, its adapters beside it
        "project-router": _projection("project", 4099, 2048, 128, 8, 4, 12, out="f32"),
        # a very small training step: launches and latency in both directions
        "tune-256": _projection("tune", 256, 512, 1024, 8, 2, 4),
        # an ordinary one, odd lengths, widths that are no multiple of a tile
        "tune-4099": _projection("tune", 4099, 2048, 1408, 16, 6, 9, bare=1),
        # a large one on the largest layer's widths and a high rank
        "tune-16384": _projection("tune", 16384, 4096, 14336, 64, 8, 16),
        # a router's loss over a very small batch
        "balance-256": _balance(256, 8, 2),
        # the benchmark layer's router
        "balance-8192": _balance(8192, 128, 8),
        # a long packed batch, a sequence each with a loss of its own, a tenth of it padding, gradient for bf16 products
        "balance-131072": _balance(131072, 256, 8, seqs=61, padding=0.1, out="bf16"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _present(c):
    """Adapters that at least one request has, on average."""
    n = c["adapters"]
    return n * (1.0 - (1.0 - 1.0 / n) ** (c["requests"] - c["bare"]))


def work(case):
    c, T = case, case["T"]
    if c["kind"] == "balance":
        dlogits = T * c["E"] * (2.0 if c["out"] == "bf16" else 4.0)
        slots = T * c["k"] * (4.0 + 8.0 * c["gates"])
        return {"bytes": 8.0 * T * c["E"] + slots + dlogits + 4.0 * T + T + 8.0 * c["seqs"] * c["E"], "flops": 0.0}
    K, N, r = c["K"], c["N"], c["rank"]
    with_adapter = T * (1.0 - c["bare"] / c["requests"])
    base, low = 2.0 * T * K * N, 2.0 * with_adapter * r * (K + N)
    factors = 2.0 * _present(c) * r * (K + N)
    tokens = 2.0 * T * K + T * N * (4.0 if c["out"] == "f32" else 2.0)
    if c["kind"] == "project":
        return {"bytes": tokens + 2.0 * K * N + factors + 4.0 * T, "flops": base + low}
    grads = 4.0 * c["adapters"] * r * (K + N)
    backward = 2.0 * T * N + 2.0 * T * K + 2.0 * T * K + 2.0 * K * N + factors + grads
    return {"bytes": tokens + 2.0 * K * N + factors + 4.0 * T + backward, "flops": 2.0 * base + 3.0 * low}


def draw(rng):
    """One more case: a kind, widths, a length and a mix of requests, all at random."""
    most = [max(work(c)[key] for c in listed()) for key in ("bytes", "flops")]

    def log(low, high):
        return round(math.exp(rng.uniform(math.log(low), math.log(high))))

    while True:
        if rng.random() < 0.25:
            E = rng.choice([8, 20, 64, 128, 129, 160, 256, 384, 512, 1000])
            T = log(64, 131072)
            c = _balance(T, E, min(E, rng.choice([1, 2, 4, 6, 8, 10, 16])), seqs=min(T, rng.choice([1, 1, log(2, 300)])),
                         padding=rng.choice([0.0, 0.0, 0.1, 0.5]), gates=rng.random() < 0.8, out=rng.choice(["f32", "f32", "bf16"]))
        else:
            kind = rng.choice(["project", "project", "tune"])
            T = rng.choice([log(1, 512), log(64, 16384)])
            adapters, requests = log(1, 256), min(T, log(1, 256))
            c = _projection(kind, T, 8 * log(8, 896), 8 * log(2, 1792), 8 * rng.choice([1, 1, 2, 2, 3, 4, 8, 16]), adapters, requests,
                            bare=rng.choice([0, 0, requests // 8]), out=rng.choice(["bf16", "bf16", "bf16", "f32"]) if kind == "project" else "bf16",
                            pad=rng.choice([0, 0, 0, 8, 64]))
            if adapters * c["rank"] * (c["K"] + c["N"]) > 1e8 or T * adapters * c["rank"] > 3e8:
                continue
        if all(work(c)[key] <= limit for key, limit in zip(("bytes", "flops"), most)):
            return c


def _normal(shape, std, g):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


def _lengths(total, parts, rng):
    """`parts` lengths of at least one that sum to `total`."""
    cuts = sorted(rng.sample(range(1, total), parts - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def prepare(case, seed):
    c, T = case, case["T"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    s = dict(c)
    if c["kind"] == "balance":
        E, k = c["E"], c["k"]
        # an uneven router: some experts are liked by every token
        logits = torch.randn((T, E), generator=g, device="cuda") + 0.7 * torch.randn((1, E), generator=g, device="cuda")
        lengths = _lengths(T, c["seqs"], rng)
        s["seq_offsets"] = None if c["seqs"] == 1 else torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
        s["mask"] = None
        if c["padding"] > 0:   # the padding stands at the sequences' ends
            keep = torch.zeros(T, dtype=torch.bool)
            at = 0
            for n in lengths:
                keep[at:at + n - int(c["padding"] * n)] = True
                at += n
            s["mask"] = keep.cuda()
        top, idx = torch.topk(logits, k, dim=1)
        s["logits"] = logits
        s["topk_idx"], s["topk_w"] = idx.to(torch.int32), torch.softmax(top, dim=1)
        s["dtopk_w"] = 1e-3 * torch.randn((T, k), generator=g, device="cuda") if c["gates"] else None
        s["dloss"] = torch.full((1,), 0.5, device="cuda")
        return s
    K, N, r, n = c["K"], c["N"], c["rank"], c["adapters"]
    adapter_of = [rng.randrange(n) for _ in range(c["requests"])]
    for i in rng.sample(range(c["requests"]), c["bare"]):
        adapter_of[i] = -1
    ids = torch.tensor(adapter_of, dtype=torch.int32)
    s["ids"] = torch.repeat_interleave(ids, torch.tensor(_lengths(T, c["requests"], rng))).cuda()
    s["x"] = _normal((T, K + c["pad"]), 1.0, g)[:, :K]
    s["w"] = _normal((K, N), 0.02, g)
    s["a"], s["b"] = _normal((n, r, K), K ** -0.5, g), _normal((n, r, N), 0.05, g)
    s["scale"] = 0.5 + 1.5 * torch.rand(n, generator=g, device="cuda")
    if c["kind"] == "tune":
        s["dy"] = _normal((T, N), 1.0, g)
    return s


def _dtype(s):
    return torch.float32 if s["out"] == "f32" else torch.bfloat16


def _own_projection(s):
    import paper_2604_19241_amd as moe
    T, K, N, r, n = s["T"], s["K"], s["N"], s["rank"], s["adapters"]
    shape = moe.make_adapter_shape(T, K, N, r, n)
    if "ws" not in s:   # kept from step to step, as every layer of these widths shares it
        s["ws"] = torch.empty(moe.moe_adapter_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    plan = moe.moe_adapter_plan(shape, s["ids"])
    if s["kind"] == "project":
        return {"y": moe.moe_adapter_forward(shape, s["x"], s["w"], s["a"], s["b"], plan, scale=s["scale"], out_dtype=_dtype(s), ws=s["ws"])}
    h = torch.empty((T, r), dtype=torch.float32, device="cuda")
    y = moe.moe_adapter_forward(shape, s["x"], s["w"], s["a"], s["b"], plan, scale=s["scale"], h=h, ws=s["ws"])
    grads = moe.moe_adapter_backward(shape, s["dy"], s["x"], s["w"], s["a"], s["b"], plan, h, scale=s["scale"], ws=s["ws"])
    return {"y": y, "dx": grads["dx"], "da": grads["da"], "db": grads["db"]}


def _own_balance(s):
    import paper_2604_19241_amd as moe
    shape = moe.make_balance_shape(s["T"], s["E"], s["k"], s["seqs"], BALANCE_COEF, Z_COEF)
    if "ws" not in s:
        s["ws"] = torch.empty(moe.moe_balance_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    stats = moe.moe_balance_forward(shape, s["logits"], s["topk_idx"], seq_offsets=s["seq_offsets"], mask=s["mask"], ws=s["ws"])
    dlogits = moe.moe_balance_backward(shape, s["logits"], s["topk_idx"], stats, seq_offsets=s["seq_offsets"],
                                       topk_w=s["topk_w"] if s["gates"] else None, dtopk_w=s["dtopk_w"], dloss=s["dloss"], out_dtype=_dtype(s))
    return {"loss": stats.loss, "counts": stats.counts, "tokens": stats.tokens, "prob_sums": stats.prob_sums, "lse": stats.lse, "dlogits": dlogits}


def _low(v, factor, ids, scale):
    """scale v factor[id]^T of every token, [T, adapters * rank]: zeros at the ranks of the adapters that are not its own."""
    n, r, width = factor.shape
    mine = (ids[:, None] == torch.arange(n, device=ids.device, dtype=ids.dtype)).float() * scale
    return ((v @ factor.reshape(n * r, width).T).view(-1, n, r) * mine[:, :, None]).view(-1, n * r)


def _plain_projection(s):
    n, r, ids, scale = s["adapters"], s["rank"], s["ids"], s["scale"]
    x, w = s["x"].float(), s["w"].float()
    if s["kind"] == "project" and s["T"] < n:   # fewer tokens than adapters: those of each token, one by one
        at = ids.clamp(min=0).long()
        h = torch.matmul(s["a"][at].float(), x[:, :, None]).transpose(1, 2) * torch.where(ids < 0, 0.0, scale[at])[:, None, None]
        return {"y": (x @ w + torch.matmul(h.contiguous(), s["b"][at].float())[:, 0]).to(_dtype(s))}
    a, b = s["a"].float(), s["b"].float()
    h = _low(x, a, ids, scale)
    y = (x @ w + h @ b.view(n * r, -1)).to(_dtype(s))
    if s["kind"] == "project":
        return {"y": y}
    dy = s["dy"].float()
    g = _low(dy, b, ids, scale)
    dx = (dy @ w.T + g @ a.view(n * r, -1)).to(torch.bfloat16)
    return {"y": y, "dx": dx, "da": (g.T @ x).view(a.shape), "db": (h.T @ dy).view(b.shape)}


def _plain_balance(s):
    T, E, k, S, logits = s["T"], s["E"], s["k"], s["seqs"], s["logits"]
    idx = s["topk_idx"].long()
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    lse = torch.where(keep, torch.logsumexp(logits, dim=1), -math.inf)
    p = torch.exp(logits - torch.logsumexp(logits, dim=1, keepdim=True)) * keep[:, None]
    seq = torch.zeros(T, dtype=torch.long, device="cuda") if S == 1 else \
        torch.searchsorted(s["seq_offsets"], torch.arange(T, device="cuda", dtype=torch.int32), right=True) - 1
    member = (seq == torch.arange(S, device="cuda")[:, None]).float() * keep
    tokens = member.sum(1)
    counts = torch.zeros(S * E, dtype=torch.int32, device="cuda")
    counts.index_add_(0, (seq[:, None] * E + idx).view(-1), keep.to(torch.int32).repeat_interleave(k))
    counts = counts.view(S, E)
    prob_sums = member @ p
    n = tokens.sum().clamp(min=1)
    f = counts / (k * tokens.clamp(min=1))[:, None]
    balance = E / n * (f * prob_sums).sum()
    z = torch.where(keep, lse, 0.0).square().sum() / n
    dloss = s["dloss"]
    fs = f[seq]
    d = dloss * BALANCE_COEF * E / n * p * (fs - (fs * p).sum(1, keepdim=True)) + \
        dloss * Z_COEF * 2 / n * torch.where(keep, lse, 0.0)[:, None] * p
    if s["gates"]:
        w, dw = s["topk_w"], s["dtopk_w"]
        d.scatter_add_(1, idx, w * (dw - (w * dw).sum(1, keepdim=True)))
    whole = torch.cat([tokens, tokens.sum()[None]]).to(torch.int32)
    return {"loss": torch.stack([BALANCE_COEF * balance + Z_COEF * z, balance, z]), "counts": counts, "tokens": whole,
            "prob_sums": prob_sums, "lse": lse, "dlogits": d.to(_dtype(s))}


def run(state):
    balance = state["kind"] == "balance"
    if own:
        return _own_balance(state) if balance else _own_projection(state)
    return _plain_balance(state) if balance else _plain_projection(state)


def _exact_projection(c, s):
    """Adapter by adapter, each merged into the projection: W + scale A^T B."""
    x, w = s["x"].double(), s["w"].double()
    tune = c["kind"] == "tune"
    out = {"y": x @ w}
    if tune:
        dy = s["dy"].double()
        out |= {"dx": dy @ w.T, "da": torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda"),
                "db": torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")}
    for i in sorted(set(s["ids"].tolist()) - {-1}):
        rows = torch.nonzero(s["ids"] == i)[:, 0]
        a, b, scale = s["a"][i].double(), s["b"][i].double(), s["scale"][i].double()
        if c["T"] < 8 * c["rank"]:
            out["y"][rows] += scale * (x[rows] @ a.T) @ b
        else:
            out["y"][rows] = x[rows] @ (w + scale * (a.T @ b))
        if tune:
            out["dx"][rows] += scale * (dy[rows] @ b.T) @ a
            outer = scale * (x[rows].T @ dy[rows])   # dL / d(A^T B)
            out["da"][i], out["db"][i] = b @ outer.T, a @ outer
    return out


def _exact_balance(c, s):
    T, E, k = c["T"], c["E"], c["k"]
    logits = s["logits"].double()
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    big = logits.max(dim=1, keepdim=True).values
    weight = torch.exp(logits - big)
    total = weight.sum(dim=1, keepdim=True)
    lse = (big + torch.log(total))[:, 0]
    p = weight / total
    starts = [0, T] if s["seq_offsets"] is None else s["seq_offsets"].tolist()
    n = int(keep.sum())
    balance, sums = 0.0, []
    d = torch.zeros_like(logits)
    dloss = float(s["dloss"])
    for lo, hi in zip(starts, starts[1:]):
        rows = torch.arange(lo, hi, device="cuda")[keep[lo:hi]]
        q = p[rows]
        sums.append(q.sum(0))
        if rows.numel() == 0:
            continue
        f = torch.bincount(s["topk_idx"][rows].long().view(-1), minlength=E).double() / (k * rows.numel())
        balance = balance + E / n * (f * sums[-1]).sum()
        slope = dloss * BALANCE_COEF * E / n * f[None] + dloss * Z_COEF * 2 / n * lse[rows][:, None]
        d[rows] = q * (slope - dloss * BALANCE_COEF * E / n * (q @ f)[:, None])
    z = lse[keep].square().sum() / max(n, 1)
    if c["gates"]:
        w, dw = s["topk_w"].double(), s["dtopk_w"].double()
        mean = (w * dw).sum(1)
        d[torch.arange(T, device="cuda")[:, None], s["topk_idx"].long()] += w * (dw - mean[:, None])
    loss = torch.stack([BALANCE_COEF * balance + Z_COEF * z, balance + 0 * z, z])
    return {"loss": loss, "counts": None, "tokens": None, "prob_sums": torch.stack(sums), "lse": torch.where(keep, lse, -math.inf), "dlogits": d}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_balance(case, s) if case["kind"] == "balance" else _exact_projection(case, s)
