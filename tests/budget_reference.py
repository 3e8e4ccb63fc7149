"""What keeps the 4-bit paged cache within a budget, in plain 64-bit arithmetic: rotary positions, attention weights of cached tokens,
which tokens are kept."""
import math

import torch

from tests import fp4_reference as ref

STEP = 2.0 ** -24           # half a step of fp32, relative


def turned(x, positions, frequencies, magnitude, interleaved, inverse=False):
    """x [rows, heads, D] -> (values, bound): the bound is what fp32 arithmetic may be off by before its result is rounded to the type.

    An angle is off by 2^-32 of a turn (its fraction is cut there), by the position times 2^-65 of a turn (the frequency's
    rounding) and by the double's here; reduced to an eighth of a turn it is rounded three times (2^-24 of 0.8 each), sine and cosine
    then by four roundings of at most 1 (the series' last steps; earlier ones count less) and their remainders, 2e-9; a product of
    them with the magnitude is rounded once more, the two products and the sum three times."""
    R = 2 * len(frequencies)
    f = torch.tensor(frequencies, dtype=torch.float64)
    p = positions.cpu().double()[:, None]
    a = p * f * (-1.0 if inverse else 1.0)
    cos, sin = torch.cos(a)[:, None] * magnitude, torch.sin(a)[:, None] * magnitude
    x = x.cpu().double()
    first, second = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    u, w = first * cos - second * sin, second * cos + first * sin
    angle = 2 * math.pi * 2.0 ** -32 + p.abs() * (2 * math.pi * 2.0 ** -65 + 2.0 ** -52 * f.abs()) + 2.0 ** -52 * a.abs()
    each = abs(magnitude) * (angle[:, None] + 2e-9 + (3 * 0.8 + 4 + 1 + 3) * STEP) * (first.abs() + second.abs())

    def joined(s, t, rest):
        y = torch.stack((s, t), -1).flatten(-2) if interleaved else torch.cat((s, t), -1)
        return torch.cat((y, rest), -1)
    return joined(u, w, x[..., R:]), joined(each, each, torch.zeros_like(x[..., R:]))


def rounded(values, bound, dtype):
    """The bound of a result rounded to dtype: half a step of it, or of the least ones."""
    info = torch.finfo(dtype)
    least = info.tiny * info.eps / 2 if dtype == torch.float16 else info.tiny   # (below it, bf16 and fp32 may be flushed)
    return bound + (values.abs() + bound) * info.eps / 2 + least


def weights(q, k, lse, n, sm_scale, window=0, sinks=0, present=None, rows=None):
    """q [n, Hq, D], k [length, H, D] (values held), lse [n, Hq] as given -> (sums [H, length], bound).  rows: which of the n count.

    Products are exact, D of them summed in fp32; the score's scaling, the scale's and the logarithm's conversion to powers of two are rounded,
    each relative to itself, their difference too; the power is off by 2^-23 of itself; sums of positive numbers in any order are
    off by a half step for each number but the first.  Powers below 2^-126 may be 0."""
    length, H, D = k.shape
    G = q.shape[1] // H
    ok = ref.seen(length, n, window, sinks)
    if present is not None:
        ok = ok & present[None, :]
    if rows is not None:
        ok = ok & rows[:, None]
    q, k, lse = q.cpu().double(), k.double(), lse.cpu().double()
    ok = ok[:, None, :] & (lse[..., None] != -math.inf)
    kk = k.repeat_interleave(G, 1)
    s = torch.einsum("nhd,thd->nht", q, kk) * sm_scale
    size = torch.einsum("nhd,thd->nht", q.abs(), kk.abs()) * abs(sm_scale)
    p = torch.where(ok, torch.exp(s - lse[..., None]), 0.0)
    off = (D + 8) * STEP * size + 3 * STEP * (s.abs() + lse.abs()[..., None]) + 2 * STEP
    sums = p.unflatten(1, (H, G)).sum((0, 2))
    bound = torch.where(ok, p * torch.expm1(off), 0.0).unflatten(1, (H, G)).sum((0, 2)) + (n * G + 1) * STEP * sums
    return sums, bound + n * G * 2.0 ** -126


def kept(mass, length, keep, sinks, recent, budget=None):
    """mass [tokens] -> positions, by going through them one by one."""
    budget = min(keep, max(budget, 0)) if budget is not None else keep
    if length <= budget:
        return list(range(length))
    sinks = min(sinks, budget)
    recent = min(recent, budget - sinks)
    order = []
    for t in range(sinks, length - recent):
        m = float(mass[t]) if t < len(mass) else 0.0
        order.append((0 if m != m else 1, -m if m == m else 0.0, t))
    order.sort()
    chosen = [t for _, _, t in order[:budget - sinks - recent]]
    return sorted(chosen + list(range(sinks)) + list(range(length - recent, length)))
