"""Moving tokens by expert, 4-bit experts and the packed stash: the workloads that their speed is followed on.

A case is one pass as a user's program makes it:

  dispatch  T tokens copied to the rows of their experts, k each, and the gradient: every token the sum of its rows';
  combine   every token the weighted sum of its rows; with `train` the gradients of the rows and of the weights too;
  rows      activations quantised to microscaled 4-bit floating point (blocks of 32 along K) and read back;
  weights   the same for the weights [K, N] of `local` experts, whose blocks run along K too;
  product   the rows of every local expert, both operands in 4 bits, by its weights (down projection);
  gate      the same gathered from T quantised tokens, by two weights: silu(x Wg) * (x Wu) (gate and up projection);
  saved     what the fused forward keeps for its backward, G and U, packed into 8 bits, and restored with h = silu(G) * U.

E experts of which k are selected for a token, the first `local` of them on this GPU.  `own` selects the framework's kernels;
otherwise the same is computed by plain torch operations in 32 bits.
"""
import math
import random

import torch

own = False

BLOCK, PAD = 32, 128   # values that share an exponent; K is filled up with zeros to a multiple of PAD


def _move(kind, T, d, E, k, local=None, type="bf16", train=True):
    return {"kind": kind, "T": T, "d": d, "E": E, "k": k, "local": E if local is None else local, "type": type, "train": train}


def _quant(kind, rows, K, N=0, type="bf16", pad=0):
    return {"kind": kind, "rows": rows, "K": K, "N": N, "type": type, "pad": pad}


def _product(kind, T, K, N, E, k, local=None, type="bf16"):
    return {"kind": kind, "T": T, "K": K, "N": N, "E": E, "k": k, "local": E if local is None else local, "type": type}


def _saved(T, I, E, k, local=None):
    return {"kind": "saved", "T": T, "I": I, "E": E, "k": k, "local": E if local is None else local}


def listed():
    cases = {
        # a very small training step: launches and latency in both directions
        "dispatch-256": _move("dispatch", 256, 512, 8, 2),
        # the benchmark layer's batch, all experts here
        "dispatch-8192": _move("dispatch", 8192, 2048, 128, 8),
        # one sequence generating: the eight expert outputs of its token
        "combine-1": _move("combine", 1, 2048, 128, 8, train=False),
        # an odd training batch in 32 bits, a quarter of the experts here
        "combine-4099": _move("combine", 4099, 2304, 256, 8, local=64, type="f32"),
        # prompts of a wide layer in front of its experts, parts of a wider buffer
        "rows-8191": _quant("rows", 8191, 7168, pad=64),
        # a layer's experts made ready for serving: its up projections
        "weights-32": _quant("weights", 32, 2048, 1408),
        # one sequence generating: eight experts' down projections, latency and the stream of the weights
        "product-1": _product("product", 1, 768, 2048, 128, 8),
        # the benchmark layer's down projections
        "product-8192": _product("product", 8192, 768, 2048, 128, 8),
        # a generation step of one rank's share of a wide layer: experts with a row or two
        "gate-37": _product("gate", 37, 7168, 2048, 256, 8, local=32),
        # prompts through few wide experts, an odd number of tokens: matrix work
        "gate-4001": _product("gate", 4001, 4096, 14336, 8, 2),
        # a short training batch's stash
        "saved-257": _saved(257, 1408, 64, 6),
        # the benchmark layer's stash
        "saved-8192": _saved(8192, 768, 128, 8),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _bytes(c):
    return 4.0 if c["type"] == "f32" else 2.0


def _codes(n, K):
    """Bytes of n rows of K values in 4 bits with their exponents."""
    return n * K * (0.5 + 1.0 / BLOCK)


def work(case):
    c, kind = case, case["kind"]
    if kind in ("rows", "weights"):
        values = float(c["rows"] * c["K"] * (c["N"] or 1))
        return {"bytes": values * (_bytes(c) + 2.0) + 2.0 * _codes(values, 1), "flops": 0.0}
    T, k = c["T"], c["k"]
    rows = T * k * c["local"] / c["E"]
    if kind == "saved":
        packed = rows * 2 * c["I"] * (1.0 + 1.0 / BLOCK)
        return {"bytes": rows * c["I"] * (4.0 + 6.0) + 2.0 * packed, "flops": 0.0}
    if kind in ("dispatch", "combine"):
        tokens, sorted_rows, slots = T * c["d"] * _bytes(c), rows * c["d"] * _bytes(c), 4.0 * T * k
        if kind == "dispatch":
            return {"bytes": 2.0 * (tokens + sorted_rows + slots), "flops": 0.0}
        back = tokens + 2.0 * sorted_rows + 3.0 * slots if c["train"] else 0.0
        return {"bytes": tokens + sorted_rows + 2.0 * slots + back, "flops": 0.0}
    pair = 2 if kind == "gate" else 1
    present = c["local"] * (1.0 - (1.0 - k / c["E"]) ** T)
    source = min(rows, float(T)) if kind == "gate" else rows
    return {"bytes": _codes(source, c["K"]) + _codes(pair * present * c["N"], c["K"]) + rows * c["N"] * _bytes(c),
            "flops": 2.0 * pair * rows * c["K"] * c["N"]}


def draw(rng):
    """One more case: a kind, a batch, a layer and a type, all at random."""
    most = [max(work(c)[key] for c in listed()) for key in ("bytes", "flops")]

    def log(low, high):
        return round(math.exp(rng.uniform(math.log(low), math.log(high))))

    while True:
        kind = rng.choice(["dispatch", "combine", "rows", "weights", "product", "product", "gate", "gate", "saved"])
        E = rng.choice([8, 20, 64, 128, 160, 256, 384, 512])
        k = rng.choice([1, 2, 4, 6, 8, 10, 16])
        local = rng.choice([E, E, max(1, E // 4), max(1, E // 8)])
        T = rng.choice([log(1, 64), log(32, 20000)])
        if k > E or T * k * local < E:   # (no row to be expected here)
            continue
        if kind in ("dispatch", "combine"):
            c = _move(kind, T, 8 * log(8, 896), E, k, local, type=rng.choice(["bf16", "bf16", "f32"]), train=kind == "dispatch" or rng.random() < 0.7)
        elif kind == "rows":
            c = _quant(kind, log(1, 20000), 8 * log(8, 1792), type=rng.choice(["bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 8, 64]))
        elif kind == "weights":
            c = _quant(kind, log(1, 128), 8 * log(8, 896), 8 * log(8, 896))
        elif kind == "saved":
            c = _saved(T, 64 * log(1, 224), E, k, local)
        else:
            c = _product(kind, T, 8 * log(8, 896), 8 * log(8, 896), E, k, local, type=rng.choice(["bf16", "bf16", "bf16", "f32"]) if kind == "product" else "bf16")
            # (the plain form holds the weights in 32 bits, and its rows filled up to the longest expert's)
            if (2 if kind == "gate" else 1) * local * c["K"] * c["N"] > 1.1e9 or T * k * max(c["K"], 2 * c["N"]) > 1.2e9:
                continue
        if all(work(c)[key] <= limit for key, limit in zip(("bytes", "flops"), most)):
            return c


def _dtype(s):
    return torch.float32 if s["type"] == "f32" else torch.bfloat16


def _routing(s, g):
    """A router's selection, an uneven one, and where its slots stand when they are sorted by expert."""
    T, E, k, local = s["T"], s["E"], s["k"], s["local"]
    logits = torch.randn((T, E), generator=g, device="cuda") + 0.3 * torch.randn((1, E), generator=g, device="cuda")
    top, idx = torch.topk(logits, k, dim=1)
    slots = idx.view(-1)
    order = torch.argsort(torch.where(slots < local, slots, E), stable=True)
    counts = torch.bincount(slots, minlength=E)[:local]
    A = int(counts.sum())
    inv = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    inv[order[:A]] = torch.arange(A, dtype=torch.int32, device="cuda")
    perm = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    perm[:A] = order[:A].to(torch.int32)
    offsets = torch.zeros(local + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    s.update(topk_idx=idx.to(torch.int32), topk_w=torch.softmax(top, dim=1), counts=counts.to(torch.int32), offsets=offsets, perm=perm,
             inv_perm=inv.view(T, k), A=A)


def _two_to(e):
    """2^e in 32 bits for whole e from -126 to 127."""
    return torch.ldexp(torch.ones((), device="cuda"), e)


def _quantized(v):
    """Codes [..., K'] (e2m1, the sign in bit 3) and exponents [..., K' / 32] of v [..., K] fp32, K' = K filled up with zeros."""
    K = v.shape[-1]
    blocks = torch.nn.functional.pad(v, (0, -K % PAD)).unflatten(-1, (-1, BLOCK))
    e = (torch.frexp(blocks.abs().amax(-1)).exponent - 1).clamp(min=-125)
    e = torch.where((blocks != 0).any(-1), e, -125)
    t = (blocks * _two_to(2 - e)[..., None]).flatten(-2)
    m = t.abs()
    code = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
    return torch.where(t < 0, code + 8, code), (e + 125).to(torch.uint8)


def _packed(v):
    """The same two to a byte, the first in the lower half."""
    code, e = _quantized(v)
    return code[..., 0::2] + 16 * code[..., 1::2], e


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _values(code, e, K):
    """What codes and exponents stand for, [..., K] fp32."""
    levels = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), device="cuda")
    scale = torch.where(e == 0, 2.0 ** -127, _two_to(e.int().clamp(min=1) - 127))
    return (levels[code.int()].unflatten(-1, (-1, BLOCK)) * scale[..., None]).flatten(-2)[..., :K]


def _unpacked(codes, e, K):
    return _values(torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2), e, K)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(c)
    kind = c["kind"]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.float32 if c.get("type") == "f32" else torch.bfloat16)

    if kind in ("rows", "weights"):
        if kind == "rows":
            # features of a residual stream: a few of them ten times the others
            loud = torch.where(torch.rand(c["K"] + c["pad"], generator=g, device="cuda") < 0.01, 10.0, 1.0)
            s["x"] = (torch.randn((c["rows"], c["K"] + c["pad"]), generator=g, device="cuda") * loud).to(_dtype(c))[:, :c["K"]]
        else:
            s["w"] = normal(c["rows"], c["K"], c["N"], std=0.02)
        return s
    _routing(s, g)
    T, k, A = c["T"], c["k"], s["A"]
    if kind in ("dispatch", "combine"):
        d = c["d"]
        # rows behind the last one stay as they are: zeros
        s["buffer"] = torch.zeros((T * k, d), dtype=_dtype(c), device="cuda")
        if kind == "dispatch":
            s["x"], s["dxs"] = normal(T, d), normal(T * k, d)
        else:
            s["o"], s["dy"] = normal(T * k, d), normal(T, d)
        return s
    if kind == "saved":
        # as the fused forward lays its stash out: G|U of every row, h, the experts' outputs (of a layer of 64 columns here)
        I = c["I"]
        sizes = [T * k * w * 2 for w in (2 * I, I, 64)]
        total = sum((n + 255) // 256 * 256 for n in sizes)
        for name in ("stash", "restored"):
            s[name] = torch.zeros(total, dtype=torch.uint8, device="cuda")
        s["gu"] = s["stash"][:sizes[0]].view(torch.bfloat16).view(T * k, 2 * I)
        s["gu"].copy_(normal(T * k, 2 * I))
        return s
    K, N, local = c["K"], c["N"], c["local"]
    s["a_codes"], s["a_scales"] = _packed(torch.randn((T if kind == "gate" else T * k, K), generator=g, device="cuda"))
    for name in ("w", "u")[:2 if kind == "gate" else 1]:
        parts = [_packed(torch.randn((N, K), generator=g, device="cuda") * K ** -0.5) for _ in range(local)]
        s[name + "_codes"], s[name + "_scales"] = (torch.stack([p[i] for p in parts]) for i in range(2))
    s["y"] = torch.zeros((T * k, N), dtype=_dtype(c), device="cuda")
    # the experts that have rows, where each row stands among its expert's, and the longest
    n = s["counts"].long()
    s["present"] = torch.nonzero(n)[:, 0]
    s["most"] = int(n.max())
    s["expert"] = torch.repeat_interleave(torch.arange(s["present"].numel(), device="cuda"), n[s["present"]])
    s["place"] = torch.arange(A, device="cuda") - torch.repeat_interleave(s["offsets"][:-1].long(), n)
    return s


# ---- the framework's kernels

def _own_moves(s):
    import paper_2604_19241_amd as moe
    shape = moe.make_dispatch_shape(s["T"], s["k"], s["d"])
    if s["kind"] == "dispatch":
        return {"xs": moe.moe_dispatch_forward(shape, s["x"], s["inv_perm"], out=s["buffer"]),
                "dx": moe.moe_dispatch_backward(shape, s["dxs"], s["inv_perm"])}
    out = {"y": moe.moe_combine_forward(shape, s["o"], s["inv_perm"], s["topk_w"])}
    if s["train"]:
        out |= moe.moe_combine_backward(shape, s["dy"], s["o"], s["inv_perm"], s["topk_w"], out={"do": s["buffer"], "dw": torch.empty_like(s["topk_w"])})
    return out


def _own_quant(s):
    import paper_2604_19241_amd as moe
    q = moe.moe_mx_quantize(s["x"]) if s["kind"] == "rows" else moe.moe_mx_quantize_weights(s["w"])
    return {"values": moe.moe_mx_values(q)}


def _own_products(s):
    import paper_2604_19241_amd as moe
    T, k, K, N = s["T"], s["k"], s["K"], s["N"]
    shape = moe.make_mx_shape(T * k, K, N, s["local"])
    a, w = moe.MXTensor(s["a_codes"], s["a_scales"], K), moe.MXTensor(s["w_codes"], s["w_scales"], K)
    if s["kind"] == "product":
        return {"y": moe.moe_mx_product(shape, a, w, s["offsets"], out_dtype=_dtype(s), y=s["y"])}
    return {"h": moe.moe_mx_gate_up(shape, a, w, moe.MXTensor(s["u_codes"], s["u_scales"], K), s["offsets"], perm=s["perm"], k=k, h=s["y"])}


def _own_saved(s):
    import paper_2604_19241_amd as moe
    shape = moe.make_shape(s["T"], 64, s["E"], s["k"], s["I"], 0, s["local"])
    routing = moe.Routing(s["topk_idx"], s["topk_w"], s["counts"], s["offsets"], s["perm"], s["inv_perm"])
    packed = moe.moe_saved_pack(shape, routing, s["stash"])
    views = moe.saved_views(shape, moe.moe_saved_unpack(shape, routing, packed, s["restored"]))
    return {"gu": views["gu"], "h": views["h"]}


# ---- plain operations

def _plain_moves(s):
    T, k, A, inv = s["T"], s["k"], s["A"], s["inv_perm"]
    order = s["perm"][:A].long()
    token, mine = order // k, (inv >= 0)[:, :, None]
    at = inv.clamp(min=0).long()
    rows = s["buffer"].clone()
    if s["kind"] == "dispatch":
        rows[:A] = s["x"][token]
        return {"xs": rows, "dx": (s["dxs"][at].float() * mine).sum(1).to(_dtype(s))}
    o, w = s["o"][at].float() * mine, s["topk_w"]
    out = {"y": (o * w[:, :, None]).sum(1).to(_dtype(s))}
    if s["train"]:
        rows[:A] = (w.view(-1)[order][:, None] * s["dy"][token].float()).to(_dtype(s))
        out |= {"do": rows, "dw": (o * s["dy"].float()[:, None]).sum(2)}
    return out


def _plain_quant(s):
    v = s["x"] if s["kind"] == "rows" else s["w"].transpose(1, 2)
    return {"values": _values(*_quantized(v.float()), s["K"]).to(torch.bfloat16)}


def _plain_products(s):
    A, K, present = s["A"], s["K"], s["present"]
    a = _unpacked(s["a_codes"], s["a_scales"], K)
    a = a[s["perm"][:A].long() // s["k"]] if s["kind"] == "gate" else a[:A]
    rows = torch.zeros((present.numel(), s["most"], K), device="cuda")
    rows[s["expert"], s["place"]] = a

    def by(name):
        w = _unpacked(s[name + "_codes"][present], s[name + "_scales"][present], K)
        return torch.bmm(rows, w.transpose(1, 2))[s["expert"], s["place"]]

    y = s["y"].clone()
    if A == 0:
        return {"y": y} if s["kind"] == "product" else {"h": y}
    if s["kind"] == "product":
        y[:A] = by("w").to(y.dtype)
        return {"y": y}
    gate = by("w")
    y[:A] = (gate / (1 + torch.exp(-gate)) * by("u")).to(y.dtype)
    return {"h": y}


def _plain_saved(s):
    A, I = s["A"], s["I"]
    blocks = s["gu"].float().unflatten(1, (-1, BLOCK))
    e = (torch.frexp(blocks.abs().amax(-1)).exponent - 1).clamp(min=-120)   # (2^(6 - e) in 32 bits)
    v = torch.round(blocks * _two_to(6 - e)[..., None]).clamp(-127, 127) * _two_to((e - 6).clamp(min=-126))[..., None]
    v = v.flatten(1)
    v[A:] = 0
    h = v[:, :I] / (1 + torch.exp(-v[:, :I])) * v[:, I:]
    return {"gu": v.to(torch.bfloat16), "h": h.to(torch.bfloat16)}


def run(state):
    kind = state["kind"]
    if kind in ("dispatch", "combine"):
        return _own_moves(state) if own else _plain_moves(state)
    if kind in ("rows", "weights"):
        return _own_quant(state) if own else _plain_quant(state)
    if kind == "saved":
        return _own_saved(state) if own else _plain_saved(state)
    return _own_products(state) if own else _plain_products(state)


# ---- the definitions in 64 bits, expert by expert and slot by slot

def _exact_moves(c, s):
    T, k, d = c["T"], c["k"], c["d"]
    inv, rows = s["inv_perm"].long(), torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
    tokens, dw = torch.zeros((T, d), dtype=torch.float64, device="cuda"), torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        t = torch.nonzero(inv[:, j] >= 0)[:, 0]
        r = inv[t, j]
        if c["kind"] == "dispatch":
            rows[r] = s["x"][t].double()
            tokens[t] += s["dxs"][r].double()
            continue
        w = s["topk_w"][t, j].double()[:, None]
        tokens[t] += w * s["o"][r].double()
        rows[r] = w * s["dy"][t].double()
        dw[t, j] = torch.linalg.vecdot(s["o"][r].double(), s["dy"][t].double())
    if c["kind"] == "dispatch":
        return {"xs": rows, "dx": tokens}
    return {"y": tokens} | ({"do": rows, "dw": dw} if c["train"] else {})


def _exact_quant(c, s):
    out = []
    for v in (s["x"].split(1024) if c["kind"] == "rows" else s["w"].transpose(1, 2)):
        v = v.double()
        K = v.shape[1]
        groups = torch.cat([v, v.new_zeros((v.shape[0], -K % BLOCK))], dim=1).view(v.shape[0], -1, BLOCK)
        top = groups.abs().amax(2, keepdim=True)
        scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2)
        t = groups / scale
        step = torch.where(t.abs() < 2, 0.5, torch.where(t.abs() < 4, 1.0, 2.0))
        out.append(((torch.round(t / step) * step).clamp(-6, 6) * scale).view(v.shape[0], -1)[:, :K])
    return {"values": torch.cat(out) if c["kind"] == "rows" else torch.stack(out)}


def _wide(codes, scales, K):
    """What stored codes stand for, from the bits of e2m1: sign, two of exponent, one of mantissa."""
    q = torch.stack([codes % 16, codes // 16], dim=-1).view(codes.shape[0], -1).double()
    sign, q = 1 - 2 * (q >= 8).double(), q % 8
    exponent, mantissa = torch.floor(q / 2), q % 2
    v = torch.where(exponent == 0, 0.5 * mantissa, torch.exp2(exponent - 1) * (1 + 0.5 * mantissa))
    return (sign * v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, dim=1))[:, :K]


def _exact_products(c, s):
    K, N, k = c["K"], c["N"], c["k"]
    y = torch.zeros((c["T"] * k, N), dtype=torch.float64, device="cuda")
    at = s["offsets"].tolist()
    for e in range(c["local"]):
        lo, hi = at[e], at[e + 1]
        if lo == hi:
            continue
        src = torch.arange(lo, hi, device="cuda") if c["kind"] == "product" else s["perm"][lo:hi].long().div(k, rounding_mode="floor")
        a = _wide(s["a_codes"][src], s["a_scales"][src], K)
        y[lo:hi] = a @ _wide(s["w_codes"][e], s["w_scales"][e], K).T
        if c["kind"] == "gate":
            y[lo:hi] *= torch.sigmoid(y[lo:hi]) * (a @ _wide(s["u_codes"][e], s["u_scales"][e], K).T)
    return {"y": y} if c["kind"] == "product" else {"h": y}


def _exact_saved(c, s):
    I, A = c["I"], s["A"]
    gu = torch.zeros((c["T"] * c["k"], 2 * I), dtype=torch.float64, device="cuda")
    h = torch.zeros((c["T"] * c["k"], I), dtype=torch.float64, device="cuda")
    for lo in range(0, A, 4096):
        v = s["gu"][lo:min(A, lo + 4096)].double()
        n = v.shape[0]
        groups = v.view(n, -1, BLOCK)
        step = torch.exp2(torch.floor(torch.log2(groups.abs().amax(2, keepdim=True).clamp(min=2.0 ** -120))) - 6)
        gu[lo:lo + n] = ((groups / step).round().clamp(-127, 127) * step).view(n, -1)
        h[lo:lo + n] = torch.nn.functional.silu(gu[lo:lo + n, :I]) * gu[lo:lo + n, I:]
    return {"gu": gu, "h": h}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("dispatch", "combine"):
        return _exact_moves(case, s)
    if kind in ("rows", "weights"):
        return _exact_quant(case, s)
    return _exact_saved(case, s) if kind == "saved" else _exact_products(case, s)
