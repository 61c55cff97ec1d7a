"""How far a decode over the 4-bit cache may be off in the mean over its outputs: bounds that follow from what its numbers are rounded
to, for ordinary data.  (The bounds of cache_reference.attention hold for any data and each output, and are wide.)"""
import torch


def rms(x):
    return x.double().pow(2).mean().sqrt().item()


def attention(q, k, v, scale, dtype=torch.float64, sink=None):
    """q [Hq][d], k, v [n][Hkv][d] -> (o [Hq][d], normalised weights [Hkv][Hq / Hkv][n]), evaluated in `dtype`."""
    hkv = k.shape[1]
    z = scale * torch.einsum("hgd,nhd->hgn", q.to(dtype).unflatten(0, (hkv, -1)), k.to(dtype))
    m = z.amax(-1, keepdim=True)
    if sink is not None:
        s = sink.to(dtype).view(hkv, -1, 1)
        m = torch.maximum(m, s)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True) + (0 if sink is None else torch.exp(s - m))
    p = p / total
    return torch.einsum("hgn,nhd->hgd", p, v.to(dtype)).flatten(0, 1), p


def bf16_bound(o, p, v):
    """rms error of a bf16 output: its own rounding, and that of the weights, which as products with their tokens' scales are
    binary16 numbers.  Each is off by 2^-11 of itself at most, and by 1/sqrt(3) of that at most in the mean; it meets a value less
    the middle of its group, half the group's range at most.  Errors of different tokens do not agree.  15 % for the spread of an
    estimate from a few thousand outputs and for all that is binary32."""
    groups = v.double().unflatten(-1, (-1, 64))
    half = (groups.amax(-1) - groups.amin(-1)) / 2                     # [n][Hkv][groups]
    weights = (2.0 ** -11 / 3 ** 0.5) ** 2 * torch.einsum("hgn,nhc->hgc", p.double() ** 2, half ** 2).mean().item()
    return 1.15 * (rms(o.to(torch.bfloat16).double() - o) ** 2 + weights) ** 0.5


def float32_bound(o, o32, p, v):
    """rms error of a float32 output.  o32: the same in torch's binary32, whose logits, exponentials and sums are rounded as often as
    the kernel's (four times that for the order of the sums and the base-2 exponential).  Weights times scales are pairs of binary16
    numbers, 22 bits, and the exponential is off by 2^-22: together 2^-21 of a weight, which meets half a group's range at most;
    twice that.  A warp adds up n / 32 sums one after another at most (torch: in a tree), each sum rounded by 2^-25 of what there is
    in the mean, at random; values and zeros apart, hence four times that."""
    groups = v.double().unflatten(-1, (-1, 64))
    half = (groups.amax(-1) - groups.amin(-1)) / 2
    weights = 2.0 ** -20 * torch.einsum("hgn,nhc->hgc", p.double() ** 2, half ** 2).mean().sqrt().item()
    return 4 * rms(o32.double() - o) + weights + 2.0 ** -23 * (len(v) / 32) ** 0.5 * rms(o)
