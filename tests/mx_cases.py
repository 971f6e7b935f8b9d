"""Microscaled 4-bit values by their definition, in 64 bits."""
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def padded(K):
    return -(-K // 128) * 128


def nibbles(codes, K):
    """Codes 0..15 [..., K], the first of a byte in its lower half."""
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2)[..., :K].long()


def values(codes, scales, K):
    """What codes and scales stand for, fp64; NaN where a scale is 255."""
    table = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device=codes.device)
    v = table[nibbles(codes, padded(K))].unflatten(-1, (-1, 32)) * torch.exp2(scales.double() - 127)[..., None]
    return torch.where((scales == 255)[..., None], float("nan"), v).flatten(-2)[..., :K]


def stand_for(x):
    """The values that x [..., K] is nearest to, ties to even, and the scales of its blocks [..., K' / 32]."""
    K = x.shape[-1]
    b = torch.nn.functional.pad(x.double(), (0, padded(K) - K)).unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2
    t = b / torch.exp2(e)[..., None]
    step = torch.where(t.abs() < 2, 0.5, torch.where(t.abs() < 4, 1.0, 2.0))
    v = ((t / step).round() * step).clamp(-6, 6) * torch.exp2(e)[..., None]
    bad = ~torch.isfinite(top)
    v = torch.where(bad[..., None], float("nan"), v)
    return v.flatten(-2)[..., :K], torch.where(bad, 255, torch.where(bad, 0.0, e) + 127).to(torch.uint8)


def same(got, want):
    """Equal as numbers, NaN where NaN."""
    nan = torch.isnan(want)
    return torch.equal(torch.isnan(got), nan) and torch.equal(torch.where(nan, 0.0, got.double()), torch.where(nan, 0.0, want))
