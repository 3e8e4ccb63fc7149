"""The 4-bit paged cache in plain 64-bit arithmetic: its values, an independent reader of its pages, and attention over it."""
import math

import torch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
PAGE, GROUP = 64, 32


def quantise(x):
    """x [..., D] -> (values, codes, exponents): for every 32 channels the least e with max |x| <= 7 * 2^e (-23 .. 13), for every
    channel the nearest magnitude, of two equally near the even code.  NaN: 0, infinities: the largest value."""
    x = torch.nan_to_num(x.double(), nan=0.0, posinf=1e30, neginf=-1e30)
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    e = torch.full(top.shape, 13, dtype=torch.int64)
    for k in range(12, -24, -1):
        e[top <= 7.0 * 2.0 ** k] = k
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64), e)[..., None]
    y = (g / scale).abs().clamp(max=6.0)
    far = (y[..., None] - MAGNITUDES).abs()
    near = far.amin(-1, keepdim=True)
    even_first = torch.where(far == near, torch.tensor([0, 8, 1, 9, 2, 10, 3, 11]), 99)   # codes 0, 2, 4, 6 before 1, 3, 5, 7
    index = even_first.argmin(-1)
    values = (MAGNITUDES[index] * scale * torch.where(torch.signbit(g), -1.0, 1.0)).flatten(-2)
    codes = (index | (torch.signbit(g).long() << 3)).flatten(-2)
    return values, codes, e


def read_page(page, head, head_dim, n_kv_heads):
    """(K, V) float64 [64, D] of a kv-head from the bytes of a page (uint8, CPU), by the layout that packkv.h states."""
    D = head_dim
    size = 64 * (D + D // 16)
    block = page.reshape(n_kv_heads, size)[head].tolist()
    signed = [m for m in MAGNITUDES.tolist()] + [-m for m in MAGNITUDES.tolist()]
    K, V = torch.zeros(64, D, dtype=torch.float64), torch.zeros(64, D, dtype=torch.float64)
    k_codes, k_scales = 0, 64 * D // 2
    v_codes, v_scales = k_scales + 2 * D, k_scales + 2 * D + 32 * D
    for t in range(64):
        for d in range(D):
            byte = block[k_codes + t * (D // 2) + d // 2]
            K[t, d] = signed[(byte >> (4 * (d % 2))) & 15] * 2.0 ** (block[k_scales + t * (D // 32) + d // 32] - 127)
            at = v_codes + 4 * ((t // 8) * D + d)
            word = int.from_bytes(bytes(block[at:at + 4]), "little")
            V[t, d] = signed[(word >> (4 * (t % 8))) & 15] * 2.0 ** (block[v_scales + (d // 32) * 64 + t] - 127)
    return K, V


def seen(length, n, window, sinks):
    """[n, length]: which tokens each of the last n rows sees."""
    p = torch.arange(length - n, length)[:, None]
    t = torch.arange(length)[None, :]
    ok = t <= p
    if window:
        ok = ok & ((t > p - window) | (t < sinks))
    return ok


def attention(q, k, v, n, sm_scale, window=0, sinks=0, present=None):
    """q [n, Hq, D], k, v [length, H, D], n and length above 0 -> (out, lse, bound, lse_bound): float64; the bounds are what an
    implementation may be off by before its result is rounded to the output's type.

    It is allowed: products of q and k exact, D of them summed in fp32 in any order (each addition off by 2^-24 of the sum of
    magnitudes), the score scaled and its exponential taken with a few roundings more; weights rounded to fp16, half a step
    2^-11 of their size (below 2^-26 of the row's largest: 2^-37 of that, half of fp16's least step 2^-24 where the largest is held as
    2^12 or more); sums over the tokens in fp32, in blocks."""
    length, H, D = k.shape
    G = q.shape[1] // H
    ok = seen(length, n, window, sinks)
    if present is not None:
        ok = ok & present[None, :]
    q, k, v = q.double(), k.double(), v.double()
    kk, vv = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    s = torch.einsum("nhd,thd->nht", q, kk) * sm_scale
    size = torch.einsum("nhd,thd->nht", q.abs(), kk.abs()) * abs(sm_scale)
    s = s.masked_fill(~ok[:, None, :], -math.inf)
    size = size.masked_fill(~ok[:, None, :], 0.0)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(s - top)
    total = w.sum(-1)
    p = w / torch.where(total > 0, total, 1.0)[..., None]
    out = torch.einsum("nht,thd->nhd", p, vv)
    lse = torch.log(total) + top[..., 0]
    # a score's error, in units of the exponent's argument; the maximum's enters the same way
    score = (D + 8) * 2.0 ** -24 * size.amax(-1) + 8 * 2.0 ** -24 * (top[..., 0].abs() + 40)
    sums = (length / 8 + 64) * 2.0 ** -24
    around = torch.einsum("nht,thd->nhd", p, vv.abs())
    bound = around * (2.0 ** -11 + 2 * score + 2 * sums)[..., None]
    bound += 2.0 ** -37 * torch.einsum("nht,thd->nhd", ok[:, None, :].double().expand_as(p), vv.abs())
    lse_bound = score + sums + 2.0 ** -21 * (1 + lse.abs())
    return out, lse, bound, lse_bound
