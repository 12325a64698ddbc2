"""Plain implementations in 64 bits of a cache in 4 bits and of attention over a
paged cache, and the tolerances of their comparisons (derived beside them)."""

from __future__ import annotations

import math

import torch

import paper_2609_20971_amd as rbs
from tests import paged_reference as R

D, BLOCK = 128, 32
STEPS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


# ------------------------------------------------------------------ 4 bits

def e2m1_encode(x):
    """x bf16 [..., d] -> codes uint8 [..., d / 2], scales uint8 [..., d / 32]."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1)
    bad = ~b.isfinite().all(-1)
    e = torch.full(top.shape, -126, dtype=torch.int64)
    finite = torch.where(bad, torch.zeros_like(top), top)
    for k in range(-126, 128):  # the least power that takes the largest under 7
        e = torch.where(finite / 2.0 ** k >= 7, torch.full_like(e, k + 1), e)
    y = torch.where(bad[..., None], torch.zeros_like(b), b) / (2.0 ** e.double())[..., None]
    far = (y.abs()[..., None] - STEPS).abs()
    near = far.amin(-1, keepdim=True)
    code = torch.where(far == near, torch.arange(8) % 2, 2).argmin(-1)  # of two as near, the even one
    code = code + 8 * torch.signbit(x).unflatten(-1, (-1, BLOCK)).long()
    code = torch.where(bad[..., None], torch.zeros_like(code), code).flatten(-2)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), scale.to(torch.uint8)


def e2m1_values(codes, scales):
    """fp64 [..., d] of codes and scales."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).long()
    y = STEPS[c & 7] * torch.where(c >= 8, -1.0, 1.0).double()
    f = torch.where(scales == 255, math.nan, 2.0 ** (scales.double() - 127))
    return (y.unflatten(-1, (-1, BLOCK)) * f[..., None]).flatten(-2)


# ------------------------------------------------------------------ caches

def make_cache(n_pages, hkv, page, fmt, layout="heads", amax=None, fill=0x5A):
    """A cache whose bytes are all `fill`."""
    def buf(width):
        if layout == "heads":
            return torch.full((n_pages, hkv, page, width), fill, dtype=torch.uint8, device="cuda")
        return torch.full((n_pages, page, hkv, width), fill, dtype=torch.uint8, device="cuda").transpose(1, 2)

    if fmt == "fp4":
        return rbs.PagedCache(buf(D // 2), buf(D // 2), None, buf(D // BLOCK), buf(D // BLOCK))
    if fmt == "fp8":
        return rbs.PagedCache(buf(D), buf(D), amax)
    return rbs.PagedCache(buf(2 * D).view(torch.bfloat16), buf(2 * D).view(torch.bfloat16))


def cache_values(cache):
    """fp64 K and V [n_pages][hkv][page][d] of a cache, on the CPU."""
    if cache.K_scale is not None:
        return [e2m1_values(c.cpu(), s.cpu()) for c, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale))]
    if cache.amax is not None:
        hkv = cache.K.shape[1]
        out = []
        for i, c in enumerate((cache.K, cache.V)):
            a = cache.amax[i * hkv:(i + 1) * hkv].cpu().double()
            out.append(R.e4m3_values(c.cpu()) * torch.where(a > 0, a / 448, torch.ones_like(a))[None, :, None, None])
        return out
    return [cache.K.cpu().double(), cache.V.cpu().double()]


def cache_of(K, V, live, fmt, layout="heads", amax=None, bad="nan"):
    """A cache that holds K and V [n_pages][hkv][page][d] where live [n_pages][page], and elsewhere NaN or the largest values."""
    def laid(x):
        return x.cuda() if layout == "heads" else x.transpose(1, 2).contiguous().cuda().transpose(1, 2)

    at = live[:, None, :, None]
    if fmt == "fp4":
        parts = []
        for x in (K, V):
            codes, scales = e2m1_encode(x.to(torch.bfloat16))
            parts.append((laid(torch.where(at, codes, 0x77).to(torch.uint8)),
                          laid(torch.where(at, scales, 255 if bad == "nan" else 0xFE).to(torch.uint8))))
        return rbs.PagedCache(parts[0][0], parts[1][0], None, parts[0][1], parts[1][1])
    if fmt == "fp8":
        hkv = K.shape[1]
        f = R.amax_factors(amax).float().view(2, 1, hkv, 1, 1)
        codes = [(x * y).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x, y in zip((K, V), f)]
        return rbs.PagedCache(*(laid(torch.where(at, x, 0x7F if bad == "nan" else 0x7E).to(torch.uint8)) for x in codes),
                              amax.cuda())
    other = torch.tensor(math.nan if bad == "nan" else math.inf, dtype=torch.bfloat16)
    return rbs.PagedCache(*(laid(torch.where(at, x.to(torch.bfloat16), other)) for x in (K, V)))


# ------------------------------------------------------------------ attention

def attend(q, k, v, scale, last, one_part=False):
    """Queries q fp64 [H_q][a][d] over keys 0 .. last[i] of k, v fp64 [H][n][d] (last < 0: none):
    O, lse and the tolerances of both.  one_part: weights held in bf16, their sum of the same."""
    hq, a = q.shape[:2]
    h, n = k.shape[:2]
    none = last < 0
    if n == 0 or bool(none.all()):
        z = torch.zeros(hq, a, dtype=torch.float64)
        return torch.zeros(hq, a, D, dtype=torch.float64), z - math.inf, torch.zeros(hq, a, D), z
    group = hq // h
    k, v = (x.repeat_interleave(group, 0) for x in (k, v))
    s = torch.matmul(q, k.transpose(1, 2)) * scale
    seen = (torch.arange(n)[None, :] <= last[:, None]) & ~none[:, None]
    s = torch.where(seen, s, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.softmax(torch.where(none[None, :, None], torch.zeros_like(s), s), -1) * (~none)[None, :, None]
    o = torch.matmul(p, v)
    # A logit: 128 products summed in fp32, then two factors, each rounded: at most 131 steps of the sum of
    # absolute products, and as much of itself.
    size = torch.where(seen, torch.matmul(q.abs(), k.abs().transpose(1, 2)) * abs(scale), 0.0).amax(-1)
    ds = size * 134 * R.U32
    logits = torch.where(seen, s.abs(), 0.0).amax(-1)
    # The exponential (argument in units of log2: a step of it, then 2 steps).
    e = ds + logits * 2 * R.U32 + 4 * R.U32
    # Weights: two bf16 parts, off by 2^-8 of a part that is 2^-8 of the weight, 2^-16; or one, off by 2^-8,
    # where the denominator sums what the products take (its lse: as far off).  Sums over n weights in fp32,
    # each partial sum below the whole one: n steps.  Joining parts: a factor (4 steps) each.
    held = 2.0 ** -8 if one_part else 2.0 ** -16
    rel = 2 * e + (n + 8) * R.U32
    mean_v = torch.matmul(p, v.abs())
    o_tol = R.HALF_BF16 * o.abs() + (mean_v * (2 * rel + 2 * held)[..., None]) * (1 + R.HALF_BF16) + 1e-38
    lse_tol = e + held + (n + 8) * R.U32 + torch.where(lse.isinf(), 0.0, lse.abs()) * 2 * R.U32
    return o, lse, o_tol, lse_tol
