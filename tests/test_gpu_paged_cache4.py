"""GPU: rows into a paged cache and out of it, and decode attention over a cache in
4 bits, against plain implementations in 64 bits (tests/cache_reference.py)."""

from __future__ import annotations

import math

import pytest
import torch

import paper_2609_20971_amd as rbs
from tests import cache_reference as C
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

D = 128
FORMATS = ["fp4", "fp8", "bf16"]


def _say(*a):
    print(*a, flush=True)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rows(n, hkv, seed):
    """bf16 [n][hkv][d] whose blocks have magnitudes of their own, with values on the borders between codes."""
    g = _gen(seed)
    x = torch.randn(n, hkv, D, generator=g) * torch.exp2(torch.randint(-20, 20, (n, hkv, 1), generator=g).float())
    x[:, :, ::17] *= 6.0
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -0.0])
    at = torch.rand(n, hkv, 4, generator=g) < 0.3
    x = x.unflatten(-1, (4, 32))
    x[..., :16] = torch.where(at[..., None], edges * torch.exp2(torch.randint(-3, 3, (n, hkv, 4, 1), generator=g).float()),
                              x[..., :16])
    x[..., 16:] = torch.where(at[..., None], x[..., 16:].clamp(-0.5, 0.5), x[..., 16:])
    return x.flatten(-2).to(torch.bfloat16)


def _laid(x, layout):
    """[n][h][d] as a (head, token, dimension) tensor of the GPU."""
    if layout == "heads":
        return x.transpose(0, 1).contiguous().cuda()
    if layout == "tokens":
        return x.contiguous().cuda().transpose(0, 1)
    wide = torch.cat([x, x * 0 + 3, x], 1).contiguous().cuda().transpose(0, 1)  # a fused projection's part
    return wide[:x.shape[1]]


def _kept(x, fmt, amax):
    """fp64 values that a cache keeps of x [n][hkv][d], and how far they may be off."""
    if fmt == "bf16":
        return x.double(), torch.zeros(x.shape, dtype=torch.float64)
    if fmt == "fp4":
        v = C.e2m1_values(*C.e2m1_encode(x))
        return v, torch.zeros_like(v)
    f = R.amax_factors(amax)[None, :, None]
    y = (x.double() * f).clamp(-448, 448)
    return y / f, (R.code_tolerance(y, torch.zeros_like(y)) + y.abs() * 4 * R.U32) / f


WRITE = [
    # tokens, kv heads, page, layouts of K, V and the cache
    (1, 1, 16, "heads", "heads", "heads"),
    (1, 4, 64, "tokens", "qkv", "tokens"),
    (3, 7, 32, "qkv", "tokens", "heads"),
    (63, 2, 16, "heads", "tokens", "tokens"),
    (65, 5, 128, "tokens", "tokens", "heads"),
    (1000, 8, 256, "qkv", "qkv", "heads"),
    (2111, 3, 16, "tokens", "heads", "tokens"),
    (4, 512, 16, "tokens", "tokens", "heads"),
    (70000, 4, 64, "tokens", "qkv", "heads"),      # 92 MB or more: past the caches
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("k", range(len(WRITE)))
def test_write_and_read_back(k, fmt):
    n, hkv, page, k_layout, v_layout, layout = WRITE[k]
    _say(f"[write] {fmt} {WRITE[k]}")
    x = [_rows(n, hkv, 2 * k + i) for i in range(2)]
    g = _gen(40 + k)
    amax = (torch.rand(2 * hkv, generator=g) * 1000 + 0.5) if fmt == "fp8" else None
    if fmt == "fp8":
        amax[0] = 0.0
    pool = -(-n // page) + 2
    order = torch.randperm(pool, generator=g)
    t = torch.arange(n)
    slots = (order[t // page] * page + t % page).to(torch.int32)
    skipped = torch.zeros(n, dtype=torch.bool)
    if n > 4:
        slots[1], slots[n - 2] = -1, pool * page
        slots[n // 2] = -2**31
        skipped[[1, n - 2, n // 2]] = True
    cache = C.make_cache(pool, hkv, page, fmt, layout, None if amax is None else amax.cuda())
    shape = rbs.make_shape(n, hkv, hkv, 64)
    K, V = _laid(x[0], k_layout), _laid(x[1], v_layout)
    assert rbs.rbs_cache_write(shape, K, V, cache, slots.cuda()) is cache
    # The cache: the written slots, and every other byte as it was.
    at = slots[~skipped].long()
    same = torch.ones(pool * page, dtype=torch.bool)
    same[at] = False
    buffers = [cache.K, cache.V] + ([cache.K_scale, cache.V_scale] if fmt == "fp4" else [])
    for b in buffers:
        b = b.contiguous().view(torch.uint8).cpu().transpose(1, 2).reshape(pool * page, -1)
        assert bool((b[same] == 0x5A).all()), "places outside the slots were written"
    for i, values in enumerate(C.cache_values(cache)):
        want, tol = _kept(x[i], fmt, None if amax is None else amax[i * hkv:(i + 1) * hkv])
        got = values[at // page, :, at % page]
        off = (got - want[~skipped]).abs()
        assert bool((off <= tol[~skipped]).all()), f"{'KV'[i]}: {float(off.max())}"
    # Read back, in the order of the tokens.
    table = order[None, :].to(torch.int32).cuda()
    k2, v2 = rbs.rbs_cache_read(shape, cache, table, _ints([0, n]))
    for i, (got, values) in enumerate(zip((k2, v2), C.cache_values(cache))):
        place = torch.arange(n)
        want = values[order[place // page], :, place % page].to(torch.bfloat16)  # (FP8: rounded once)
        got = got.cpu().transpose(0, 1)
        if fmt == "fp8":
            off = (got.double() - want.double()).abs()[~skipped]  # a factor and two roundings, and the bf16 step that they may cross
            assert bool((off <= want.double().abs()[~skipped] * 2 ** -7).all())
        else:
            assert torch.equal(got[~skipped], want[~skipped])


def test_fp4_extreme_values():
    """NaN and infinities make their own 32 elements NaN; zeros, the least and the largest magnitudes."""
    x = _rows(12, 2, 3)
    x[0] = 0.0
    x[1, 0, 5] = math.nan
    x[2, 1, 64] = math.inf
    x[3, 0, 127] = -math.inf
    x[4] = 3.38e38
    x[5] = torch.tensor(1e-40).to(torch.bfloat16)      # subnormal
    x[6] = torch.exp2(torch.tensor(-126.0))
    x[7, 0, :32] = 7.0
    x[7, 1, :32] = 6.96875                               # the last below 7
    x[8, 0] = -0.0
    x[9, 0, 40] = math.nan
    x[9, 0, 41] = math.inf
    cache = C.make_cache(1, 2, 16, "fp4")
    n = x.shape[0]
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    shape = rbs.make_shape(n, 2, 2, 64)
    rbs.rbs_cache_write(shape, _laid(x, "tokens"), _laid(x, "heads"), cache, slots)
    codes, scales = C.e2m1_encode(x)
    for c, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        assert torch.equal(c[0, :, :n].cpu().transpose(0, 1), codes)
        assert torch.equal(s[0, :, :n].cpu().transpose(0, 1), scales)
    k, v = rbs.rbs_cache_read(shape, cache, _ints([[0]]), _ints([0, n]))
    want = C.e2m1_values(codes, scales).to(torch.bfloat16)
    for got in (k, v):
        got = got.cpu().transpose(0, 1)
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(5.0), want.nan_to_num(5.0))
    assert int(want.isnan().sum()) == 4 * 32


def test_scales_of_any_byte_are_read():
    """A cache written elsewhere may hold any scale: 0 is 2^-127, and past the largest magnitude comes an infinity."""
    g = _gen(8)
    codes = torch.randint(0, 256, (256, 1, 16, D // 2), generator=g, dtype=torch.uint8)
    scales = torch.arange(256, dtype=torch.uint8)[:, None, None, None].expand(256, 1, 16, 4).contiguous()
    cache = rbs.PagedCache(codes.cuda(), codes.cuda(), None, scales.cuda(), scales.cuda())
    n = 256 * 16
    k, _ = rbs.rbs_cache_read(rbs.make_shape(n, 1, 1, 64), cache, torch.arange(256, dtype=torch.int32, device="cuda")[None],
                              _ints([0, n]))
    want = C.e2m1_values(codes, scales).to(torch.bfloat16).reshape(n, D)
    assert torch.equal(k[0].cpu().nan_to_num(5.0), want.nan_to_num(5.0))


READ = [
    # lengths of the packed rows, starts, page, capacity to spare
    ([5], [0], 16, 0),
    ([1, 0, 40, 0, 0, 17], [3, 9, 15, 0, 1, 100], 16, 6),
    ([64] * 9, [1] * 9, 64, 1),
    ([700, 1, 333], [5, 0, 255], 256, 70),
    ([3] * 4096, [7] * 4096, 32, 5),
    ([0] * 30 + [2000] + [0] * 30, [11] * 61, 128, 0),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("k", range(len(READ)))
def test_read_rows(k, fmt):
    counts, starts, page, spare = READ[k]
    hkv, n_rows = 3, len(counts)
    _say(f"[read] {fmt} rows {n_rows} page {page}")
    g = _gen(60 + k)
    columns = max(-(-(s + c) // page) for s, c in zip(starts, counts)) + 1
    pool = 50
    table = torch.randint(0, pool, (n_rows, columns), generator=g, dtype=torch.int32)  # (rows may share pages)
    K, V = (torch.randn(pool, hkv, page, D, generator=g) for _ in range(2))
    amax = torch.rand(2 * hkv, generator=g) * 3 + 2
    cache = C.cache_of(K, V, torch.ones(pool, page, dtype=torch.bool), fmt, "tokens", amax)
    total = sum(counts)
    n = total + spare
    cu = [0]
    for c in counts:
        cu.append(cu[-1] + c)
    out = [torch.full((n, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1) for _ in range(2)]
    got = rbs.rbs_cache_read(rbs.make_shape(n, hkv, hkv, 64), cache, table.cuda(), _ints(cu), _ints(starts), *out)
    assert got[0] is out[0] and got[1] is out[1]
    row = torch.repeat_interleave(torch.arange(n_rows), torch.tensor(counts))
    p = torch.arange(total) - torch.tensor(cu)[row] + torch.tensor(starts)[row]
    for got, values in zip(out, C.cache_values(cache)):
        want = values[table[row, p // page].long(), :, p % page]
        got = got.cpu().transpose(0, 1)
        assert bool((got[total:] == 7.0).all()), "tokens of no row were written"
        off = (got[:total].double() - want).abs()
        tol = want.abs() * (R.HALF_BF16 + 2 * R.U32) if fmt == "fp8" else 0 * want
        assert bool((off <= tol).all())


def test_read_outside_the_table():
    """Positions outside the row's table are left alone, page numbers outside the cache clamped; odd offsets write nothing."""
    g = _gen(5)
    K, V = (torch.randn(4, 2, 16, D, generator=g) for _ in range(2))
    cache = C.cache_of(K, V, torch.ones(4, 16, dtype=torch.bool), "fp4")
    table = _ints([[1, 2], [2**31 - 1, -2**31]])
    shape = rbs.make_shape(40, 2, 2, 64)

    def read(cu, starts):
        out = [torch.full((2, 40, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        rbs.rbs_cache_read(shape, cache, table, _ints(cu), _ints(starts), *out)
        return out[0].cpu()

    values = C.cache_values(cache)[0].to(torch.bfloat16)
    got = read([0, 20, 40], [-5, 25])
    assert bool((got[:, :5] == 7.0).all()) and torch.equal(got[:, 5:20], values[1, :, :15])
    assert torch.equal(got[:, 20:27], values[0, :, 9:16]) and bool((got[:, 27:] == 7.0).all())
    got = read([0, 16, 16], [0, 0])
    assert torch.equal(got[:, :16], values[1]) and bool((got[:, 16:] == 7.0).all())
    assert torch.equal(read([0, 0, 16], [0, 2**31 - 1]), torch.full_like(got, 7.0))
    read([-2**31, 2**31 - 1, -7], [2**31 - 1, -2**31])  # (in bounds whatever they hold)


def test_same_as_the_norm_and_rotation_call():
    """A cache in 4 bits written by rbs_qk_norm_rope holds what rbs_cache_write makes of its K_out, bit for bit."""
    for k, (n, hq, hkv, rot, interleaved, page, layout) in enumerate([
            (1, 8, 4, 128, False, 16, "heads"), (37, 7, 7, 128, True, 32, "tokens"), (70, 4, 2, 64, False, 16, "heads"),
            (70, 4, 2, 8, False, 64, "heads"), (70, 4, 2, 8, True, 64, "heads"), (41, 6, 3, 120, False, 16, "tokens"),
            (41, 6, 3, 0, False, 16, "heads"), (333, 5, 1, 96, True, 256, "tokens"), (333, 5, 1, 40, False, 256, "tokens"),
            (4111, 64, 8, 128, False, 16, "heads"), (4111, 64, 8, 96, True, 128, "tokens"),  # past the caches, runs of eight
            (4111, 64, 8, 72, False, 64, "heads")]):
        _say(f"[rope, 4 bits] {n} tokens, {hq}/{hkv}, {rot} rotated")
        g = _gen(100 + k)
        qkv = (torch.randn(n, hq + 2 * hkv, D, generator=g) * 1.5).to(torch.bfloat16)
        qkv[:, :, 5::31] *= 5
        qkv = qkv.cuda().transpose(0, 1)
        Q, K, V = qkv[:hq], qkv[hq:hq + hkv], qkv[hq + hkv:]
        w = (1 + 0.3 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda()
        inv, factor = rbs.rope_frequencies(rot) if rot else (None, 1.0)
        rope = rbs.Rope(inv, w, w, interleaved=interleaved, factor=factor)
        pos = torch.randint(0, 131072, (n,), generator=g, dtype=torch.int32).cuda()
        pool = -(-n // page) + 1
        slots = torch.randperm(pool * page, generator=g)[:n].to(torch.int32)
        if n > 2:
            slots[2] = -1
        shape = rbs.make_shape(n, hq, hkv, 64)
        fused, apart = (C.make_cache(pool, hkv, page, "fp4", layout) for _ in range(2))
        _, k_out = rbs.rbs_qk_norm_rope(shape, rope, Q, K, pos, V=V, cache=fused, slots=slots.cuda())
        rbs.rbs_cache_write(shape, k_out, V, apart, slots.cuda())
        for name in ("K", "V", "K_scale", "V_scale"):
            assert torch.equal(getattr(fused, name), getattr(apart, name)), name


# ------------------------------------------------------------------ decode

def _case(lens, hq, hkv, page, layout, seed, fmt="fp4", columns=1, bad="nan", k_scale=1.0):
    g = _gen(seed)
    n = len(lens)
    held = [-(-max(x, 0) // page) for x in lens]
    columns, pool = max(1, max(held)) + columns, sum(held) + 2
    order = torch.randperm(pool, generator=g).tolist()
    table = torch.full((n, columns), -123456, dtype=torch.int32)
    live = torch.zeros(pool, page, dtype=torch.bool)
    for row, x in enumerate(lens):
        for j in range(held[row]):
            table[row, j] = order.pop()
            live[table[row, j], :min(page, x - j * page)] = True
    K = torch.randn(pool, hkv, page, D, generator=g) * k_scale + 0.3 * torch.randn(1, hkv, 1, D, generator=g)
    K = K * torch.exp2(torch.randint(-4, 3, (1, hkv, 1, 4), generator=g).float()).repeat_interleave(32, -1)
    V = torch.randn(pool, hkv, page, D, generator=g) * torch.exp2(torch.randint(-3, 3, (pool, 1, page, 1), generator=g).float())
    q = (torch.randn(n, hq, D, generator=g) * 1.5).to(torch.bfloat16)
    amax = torch.rand(2 * hkv, generator=g) * 3 + 2
    cache = C.cache_of(K, V, live, fmt, layout, amax, bad)
    return dict(cache=cache, table=table, lens=lens, q=q, page=page, hq=hq, hkv=hkv, n=n, fmt=fmt)


def _run(c, scale=0.0, q_layout="tokens", lse=True, **more):
    Q = _laid(c["q"], q_layout)
    O = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device="cuda").fill_(math.nan)
    l = torch.full((c["hq"], c["n"]), math.nan, device="cuda") if lse else None
    got = rbs.rbs_paged_decode(rbs.make_shape(c["n"], c["hq"], c["hkv"], 64), Q, c["cache"], c["table"].cuda(), _ints(c["lens"]),
                               scale, O=O, lse=l, **more)
    assert got is O
    return O, l


def _check(c, O, lse, scale):
    K, V = C.cache_values(c["cache"])
    worst = 0.0
    for row, n in enumerate(c["lens"]):
        if n < 0:
            assert bool(O[:, row].isnan().all()), f"unused row {row} was written"
            continue
        k, v = (R.gather(x, c["table"][row], n, c["page"]) for x in (K, V))
        o, l, o_tol, l_tol = C.attend(c["q"][row].double()[:, None], k, v, scale, torch.tensor([n - 1]))
        err = (O[:, row].cpu().double() - o[:, 0]).abs()
        assert bool((err <= o_tol[:, 0]).all()), f"row {row} of length {n}: {(err / o_tol[:, 0]).max():.3f} of the tolerance"
        if n > 0:
            worst = max(worst, float((err / o_tol[:, 0]).max()))
        if lse is not None:
            got = lse[:, row].cpu().double()
            assert bool(((got - l[:, 0]).abs() <= l_tol[:, 0]).all() if n > 0 else (got == -math.inf).all()), f"row {row}: lse"
    return worst


DECODE = [
    # lengths, heads, page, cache layout, q layout, scale
    ([1], 2, 1, 16, "heads", "heads", 0.0),
    ([1, 0, 2, 15, 16, 17, -1, 31, 32, 33, 63, 64, 65], 8, 2, 16, "tokens", "tokens", 0.0),
    ([127, 128, 129, 511, 1000], 7, 1, 32, "heads", "qkv", 0.3),
    ([700], 32, 4, 16, "heads", "tokens", 0.0),
    ([769], 16, 2, 64, "heads", "tokens", 0.0),
    ([5000, 3, 2047], 28, 4, 128, "tokens", "tokens", 0.0),
    ([257] * 3, 17, 1, 256, "heads", "heads", 0.0),          # two columns of query heads
    ([300, 40], 66, 2, 64, "heads", "tokens", 0.0),
    ([(i * 53) % 260 for i in range(700)], 16, 8, 16, "heads", "tokens", 0.0),     # a wave to a row
    ([150] * 520 + [2500] * 3, 16, 1, 16, "heads", "tokens", 0.0),                 # more rows than workers
    ([6000] * 40 + [0, 33, -1], 16, 8, 16, "tokens", "tokens", 0.0),                # past the caches
    ([70] + [0] * 2000 + [-1] * 2000 + [3000, 33], 8, 2, 16, "heads", "tokens", 0.0),
    ([512, 3000], 512, 512, 16, "heads", "tokens", 0.0),
    ([150001], 8, 1, 64, "heads", "tokens", 0.0),
]


@pytest.mark.parametrize("k", range(len(DECODE)))
def test_decode(k):
    lens, hq, hkv, page, layout, q_layout, scale = DECODE[k]
    _say(f"[decode, 4 bits] {len(lens)} rows, heads {hq}/{hkv}, page {page}")
    c = _case(lens, hq, hkv, page, layout, 200 + k)
    O, lse = _run(c, scale, q_layout)
    _say(f"[decode, 4 bits] {_check(c, O, lse, scale if scale > 0 else 1 / math.sqrt(D)):.3f} of the tolerance")
    O2, _ = _run(c, scale, q_layout, lse=False)
    assert torch.equal(O.nan_to_num(9.0), O2.nan_to_num(9.0)), "the same call again"


def test_decode_large_logits_and_places_past_the_length():
    c = _case([700, 33, 5000], 8, 2, 16, "heads", 91, bad="large", k_scale=12.0)
    O, lse = _run(c, 2.0)
    _check(c, O, lse, 2.0)


def test_decode_query_magnitudes():
    """Query rows of any magnitude, with elements far below their largest; a row that is not finite is its own."""
    c = _case([300, 301, 302, 303, 304, 305], 8, 2, 16, "heads", 95)
    q = c["q"]
    q[0] *= 2.0 ** -40
    q[1, :, ::2] *= 2.0 ** -16
    q[2] = 0
    q[3, 0] *= 2.0 ** -130          # subnormal
    q[3, 1] *= 2.0 ** 60
    O, lse = _run(c, 2.0 ** -8)
    _check(c, O, lse, 2.0 ** -8)
    clean = O.clone()
    q[4, 3, 7], q[5, 6, 127] = math.nan, math.inf
    O, _ = _run(c, 2.0 ** -8)
    assert bool(O[3, 4].isnan().all()) and bool(O[6, 5].isnan().all())
    keep = torch.ones(8, 6, dtype=torch.bool)
    keep[3, 4] = keep[6, 5] = False
    assert torch.equal(O[keep.cuda()], clean[keep.cuda()])


@pytest.mark.parametrize("other", [1, 3, 20, 40, 127])
def test_decode_small_products_beside_large_ones(other):
    """One key: a product of 16 and one of 2^-n, of elements next to each other and apart."""
    n = 20
    cache = rbs.PagedCache.allocate(n, 16, 1, fp4=True)
    for t in (cache.K, cache.V):
        t.zero_()
    for t in (cache.K_scale, cache.V_scale):
        t.fill_(127)
    q, k = torch.zeros(n, D), torch.zeros(n, D)
    q[:, 0], q[:, other] = 4.0, 2.0 ** -torch.arange(n)
    k[:, 0], k[:, other] = 4.0, 1.0
    codes, scales = C.e2m1_encode(k.to(torch.bfloat16))
    cache.K[:, 0, 0], cache.K_scale[:, 0, 0] = codes.cuda(), scales.cuda()
    lse = torch.empty(1, n, device="cuda")
    rbs.rbs_paged_decode(rbs.make_shape(n, 1, 1, 64), q.to(torch.bfloat16).cuda()[None], cache,
                         torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous(), _ints([1] * n), 1.0, lse=lse)
    want = (q * k).double().sum(-1)
    # The sum, two factors (log2 e and ln 2, each rounded too) and the result: 6 steps.
    assert bool(((lse[0].cpu().double() - want).abs() <= 6 * R.U32 * want).all())


def test_decode_nan_in_attended_places():
    """A NaN key or value reaches its own head's rows only."""
    c = _case([100, 200], 8, 2, 16, "heads", 96)
    clean, _ = _run(c)
    page, place = int(c["table"][0, 3]), 5
    c["cache"].K_scale[page, 0, place, 2] = 255
    c["cache"].V_scale[page, 1, place, 1] = 255
    O, _ = _run(c)
    assert bool(O[:4, 0].isnan().all())
    assert bool(O[4:, 0, 32:64].isnan().all()) and not bool(O[4:, 0, :32].isnan().any())
    assert torch.equal(O[:, 1], clean[:, 1]) and torch.equal(O[4:, 0, 64:], clean[4:, 0, 64:])


def test_decode_clamps_lengths_and_pages():
    c = _case([64, 64], 4, 2, 16, "heads", 93, columns=0)
    want, _ = _run(c)
    got, _ = _run(dict(c, lens=[2**31 - 1, 64]))
    assert torch.equal(got, want)
    pool = c["cache"].K.shape[0]
    wild, tame = (dict(c, table=c["table"].clone()) for _ in range(2))
    wild["table"][0, 1], wild["table"][0, 2] = 2**31 - 1, -2**31
    tame["table"][0, 1], tame["table"][0, 2] = pool - 1, 0
    assert torch.equal(_run(wild)[0].nan_to_num(3.0), _run(tame)[0].nan_to_num(3.0))


def test_pages_past_32_bits():
    """A cache of more than 2^32 bytes of codes a tensor: written, read and attended in its last pages as in a small one."""
    page, hkv, hq = 256, 8, 16
    n_pages = (1 << 33) // (page * hkv * D) + 40
    c = _case([5000, 300], hq, hkv, page, "heads", 94)
    small = c["cache"].K.shape[0]
    far = rbs.PagedCache.allocate(n_pages, page, hkv, fp4=True)
    assert far.K.numel() > 1 << 32
    for name in ("K", "V", "K_scale", "V_scale"):
        getattr(far, name)[-small:] = getattr(c["cache"], name)
    moved = dict(c, cache=far, table=torch.where(c["table"] >= 0, c["table"] + n_pages - small, c["table"]))
    want, got = _run(c), _run(moved)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    x = _rows(4, hkv, 97)
    slots = _ints([(n_pages - 1) * page + 255, (n_pages - 3) * page, 7, -1])
    shape = rbs.make_shape(4, hkv, hkv, 64)
    rbs.rbs_cache_write(shape, _laid(x, "tokens"), _laid(x, "heads"), far, slots)
    k, v = rbs.rbs_cache_read(rbs.make_shape(3, hkv, hkv, 64), far, _ints([[n_pages - 1], [n_pages - 3], [0]]),
                              _ints([0, 1, 2, 3]), _ints([255, 0, 7]))
    want = C.e2m1_values(*C.e2m1_encode(x))[:3].to(torch.bfloat16)
    assert torch.equal(k.cpu().transpose(0, 1), want) and torch.equal(v.cpu().transpose(0, 1), want)


def test_strided_buffers():
    """Keys and values in one buffer, rows with room between them, and one page or head of any stride."""
    hkv, page, pool = 2, 16, 5
    codes = torch.full((pool, 2, page, hkv + 1, D // 2), 0x33, dtype=torch.uint8, device="cuda")
    scales = torch.full((pool, 2, page, hkv + 1, D // 32), 0x33, dtype=torch.uint8, device="cuda")
    parts = [x[:, i].transpose(1, 2)[:, :hkv] for x in (codes, scales) for i in range(2)]
    cache = rbs.PagedCache(parts[0], parts[1], None, parts[2], parts[3])
    plain = C.make_cache(pool, hkv, page, "fp4")
    x, y = _rows(60, hkv, 11), _rows(60, hkv, 12)
    slots = torch.randperm(pool * page, generator=_gen(1))[:60].to(torch.int32).cuda()
    shape = rbs.make_shape(60, hkv, hkv, 64)
    for to in (cache, plain):
        rbs.rbs_cache_write(shape, _laid(x, "tokens"), _laid(y, "qkv"), to, slots)
    at = slots.long()
    for name in ("K", "V", "K_scale", "V_scale"):
        a, b = (getattr(z, name)[at // page, :, at % page] for z in (cache, plain))
        assert torch.equal(a, b)
    assert bool((codes[:, :, :, hkv] == 0x33).all()) and bool((scales[:, :, :, hkv] == 0x33).all())
    table = torch.arange(pool, dtype=torch.int32, device="cuda")[None]
    q = torch.randn(4, 1, D, generator=_gen(2)).to(torch.bfloat16).cuda()
    length = _ints([60])
    for b in (cache, plain):  # (places that were not written: 0x33 and 0x5A, finite in both)
        b.K.copy_(cache.K), b.V.copy_(cache.V), b.K_scale.copy_(cache.K_scale), b.V_scale.copy_(cache.V_scale)
    shape = rbs.make_shape(1, 4, hkv, 64)
    assert torch.equal(rbs.rbs_paged_decode(shape, q, cache, table, length), rbs.rbs_paged_decode(shape, q, plain, table, length))
