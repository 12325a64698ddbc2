"""Plain implementations in 64 bits of the calls over a paged cache, and the
tolerances of their comparisons (derived beside them)."""

from __future__ import annotations

import math

import torch

D = 128
E4M3_MAX = 448.0
HALF_BF16, U32 = 2.0 ** -8, 2.0 ** -24  # half a step of bf16, of fp32, relative to the value


# ------------------------------------------------------------------ pages

def extend(table, free, n_free, lens, new, page, max_tokens):
    """One token after another; lists in, a dict of lists out (table: a copy)."""
    add = [0 if n < 0 else max(0, a) for n, a in zip(lens, new)]
    need = [-(-(n + a) // page) - -(-n // page) if n >= 0 else 0 for n, a in zip(lens, add)]
    status = (1 if sum(need) > max(0, n_free) else 0)
    status |= 2 if any(n >= 0 and -(-(n + a) // page) > len(table[0]) for n, a in zip(lens, add)) else 0
    status |= 4 if sum(add) > max_tokens else 0
    status |= 8 if not 0 <= n_free <= len(free) else 0
    table, stack = [list(r) for r in table], list(free[:max(0, n_free)])
    out = dict(table=table, n_free=n_free, lens=list(lens), cu=[0] * (len(lens) + 1), positions=[-1] * max_tokens,
               slots=[-1] * max_tokens, status=status)
    if status:
        return out
    t = 0
    for row, a in enumerate(add):
        for p in range(lens[row], lens[row] + a):
            if p % page == 0:
                table[row][p // page] = stack.pop()
            out["positions"][t] = p
            out["slots"][t] = table[row][p // page] * page + p % page
            t += 1
        out["lens"][row] += a
        out["cu"][row + 1] = t
    out["n_free"] = len(stack)
    return out


# ------------------------------------------------------------------ norm and rotation

def e4m3_values(codes):
    """fp64 values of uint8 E4M3 codes (bias 7, 3 bits of mantissa)."""
    c = codes.long()
    sign = torch.where(c >= 128, -1.0, 1.0).double()
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.pow(2.0, (e - 7).double()))
    return sign * torch.where((c & 127) == 127, torch.full_like(v, math.nan), v)


def amax_factors(amax):
    """What a value is multiplied by to become a code's, per head."""
    a = amax.double()
    return torch.where(a > 0, E4M3_MAX / a, torch.ones_like(a))


def norm_rope(x, positions, inv_freq, weight, eps, interleaved, factor):
    """x fp64 [H][T][d]; (result, |a| + |b| of each element's pair: the scale of its fp32 errors)."""
    y = x
    if weight is not None:
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    out, size = y.clone(), y.abs().clone()
    if rot:
        a_at = torch.arange(rot // 2) * 2 if interleaved else torch.arange(rot // 2)
        b_at = a_at + (1 if interleaved else rot // 2)
        angle = positions.double()[:, None] * inv_freq.double()
        cos, sin = torch.cos(angle) * factor, torch.sin(angle) * factor
        a, b = y[..., a_at], y[..., b_at]
        out[..., a_at], out[..., b_at] = a * cos - b * sin, b * cos + a * sin
        size[..., a_at] = size[..., b_at] = (a.abs() + b.abs()) * abs(factor)
    return out, size


# fp32 steps before the one rounding: the mean square (128 products and sums, at
# most 130 roundings; half of them after the square root), the division and the
# two factors (4), sine and cosine (2 steps each, and the fraction of a turn, up
# to 2^-25 of a turn: 2 pi 2^-25 < 4 U32), the rotation (3): under 90 steps of U32.
ROPE_F32 = 90 * U32


def bf16_tolerance(exact, size):
    return HALF_BF16 * exact.abs() + size * ROPE_F32 * (1 + HALF_BF16) + 1e-38


def code_tolerance(exact, size):
    """In units of the codes: half a step of E4M3 (2^-4 of the value; 2^-10 where it is subnormal)."""
    return torch.maximum(exact.abs() * 2.0 ** -4, torch.full_like(exact, 2.0 ** -10)) + size * (ROPE_F32 + 4 * U32) * 1.1


# ------------------------------------------------------------------ attention

def gather(cache, table_row, length, page):
    """[n_pages][H][page][d] -> [H][length][d]."""
    pages = table_row[:-(-length // page)].long()
    x = cache[pages].transpose(0, 1)
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :length]


def attend(q, k, v, scale):
    """q fp64 [H_q][d], k, v fp64 [H][n][d] -> O, lse, and the tolerances of both."""
    hq, (h, n) = q.shape[0], k.shape[:2]
    if n == 0:
        zero = torch.zeros(hq, dtype=torch.float64)
        return torch.zeros(hq, D, dtype=torch.float64), zero - math.inf, torch.zeros(hq, D), zero
    qg = q.view(h, hq // h, D)
    s = torch.matmul(qg, k.transpose(1, 2)) * scale
    lse = torch.logsumexp(s, -1)
    p = torch.softmax(s, -1)
    o = torch.matmul(p, v)
    # A logit: 128 products summed in fp32, then two factors, each rounded: at
    # most 131 steps of the sum of absolute products, and as much of itself.
    ds = (torch.matmul(qg.abs(), k.abs().transpose(1, 2)) * abs(scale)).amax(-1) * 134 * U32
    # The exponential (argument in units of log2: a step of it, then 2 steps).
    e = ds + s.abs().amax(-1) * 2 * U32 + 4 * U32
    # Weights held as two bf16 parts: off by 2^-8 of a part that is 2^-8 of the
    # weight, 2^-16.  Sums over n weights in fp32, each partial sum below the
    # whole one: n steps.  Joining parts: a factor (4 steps) each.
    rel = 2 * e + 2.0 ** -16 + (n + 8) * U32
    mean_v = torch.matmul(p, v.abs())
    o_tol = HALF_BF16 * o.abs() + (mean_v * 2 * rel[..., None]) * (1 + HALF_BF16) + 1e-38
    lse_tol = e + 2.0 ** -16 + (n + 8) * U32 + lse.abs() * 2 * U32
    return o.reshape(hq, D), lse.reshape(hq), o_tol.reshape(hq, D), lse_tol.reshape(hq)
