"""GPU: the calls over a paged key-value cache against plain implementations in
64 bits (tests/paged_reference.py, where the tolerances are derived)."""

from __future__ import annotations

import math

import pytest
import torch

import paper_2609_20971_amd as rbs
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

D = 128


def _say(*a):
    print(*a, flush=True)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------ pages

def _pages(lens, page, columns, pool, seed, spare=None):
    """Pages whose rows hold distinct random pages for the given lengths."""
    order = torch.randperm(pool, generator=_gen(seed)).tolist()
    table = [[-7] * columns for _ in lens]
    for row, n in enumerate(lens):
        for j in range(-(-n // page) if n > 0 else 0):
            table[row][j] = order.pop()
    free = order + [-9] * (pool - len(order))
    n_free = len(order) if spare is None else spare
    return table, free, n_free


EXTEND = [
    # lengths, new tokens (None: one each), page, columns, pages to spare, capacity to spare
    ([0], [1], 16, 1, 0, 0),
    ([0], [0], 16, 1, 3, 5),
    ([16], None, 16, 2, 0, 0),
    ([15, 16, 17, -1, 0, 31], None, 16, 4, 2, 3),
    ([5, -1, 0, 200, -3], [100, 50, 33, 0, -4], 32, 10, 1, 0),
    ([0] * 40, [777] * 40, 64, 13, 7, 2),                      # 31080 tokens: eight workgroups
    ([1] * 1025, None, 16, 1, 0, 1),                            # two rows a thread
    ([(37 * i) % 300 - 1 for i in range(4096)], None, 128, 3, 9, 0),
    ([(37 * i) % 300 for i in range(3000)], [(11 * i) % 7 - 1 for i in range(3000)], 256, 2, 1, 11),
    ([9] * 4096, [3] + [0] * 2000 + [1] + [0] * 2093 + [2500], 64, 41, 4, 6),               # few rows take tokens
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("k", range(len(EXTEND)))
def test_extend(k, in_place):
    lens, new, page, columns, spare, room = EXTEND[k]
    counts = [1] * len(lens) if new is None else new
    add = [max(0, a) if n >= 0 else 0 for n, a in zip(lens, counts)]
    held = sum(-(-n // page) for n in lens if n > 0)
    need = sum(-(-(n + a) // page) for n, a in zip(lens, add) if n >= 0) - held
    _run_extend(lens, new, page, columns, held + need + spare, max(1, sum(add) + room), in_place, want_status=0)


def _run_extend(lens, new, page, columns, pool, max_tokens, in_place, want_status, n_free=None):
    table, free, n_free = _pages(lens if n_free is None else [0] * len(lens), page, columns, pool, 5, n_free)
    _say(f"[extend] rows {len(lens)} page {page} pool {pool} tokens {max_tokens} in place {in_place}")
    pages = rbs.Pages(_ints(table), _ints(free), _ints([n_free]), _ints(lens), page)
    step = rbs.PageStep.allocate(pages, max_tokens, in_place=in_place)
    rbs.rbs_pages_extend(pages, None if new is None else _ints(new), step=step)
    want = R.extend(table, free, n_free, lens, [1] * len(lens) if new is None else new, page, max_tokens)
    assert want["status"] == want_status
    assert step.status.tolist() == [want["status"]]
    assert step.seq_lens.tolist() == want["lens"]
    assert step.n_free.tolist() == [want["n_free"]]
    assert step.cu_tokens.tolist() == want["cu"]
    assert step.positions.tolist() == want["positions"]
    assert step.slots.tolist() == want["slots"]
    assert pages.page_table.tolist() == want["table"]
    assert pages.free_pages.tolist() == free
    if not in_place:
        assert pages.seq_lens.tolist() == lens and pages.n_free.tolist() == [n_free]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lens,new,page,columns,pool,max_tokens,n_free,status", [
    ([16, 16], None, 16, 4, 3, 2, None, 1),                         # one free page, two needed
    ([0, 60], [1, 5], 16, 4, 9, 6, None, 2),                        # row 1 would take a fifth page
    ([0, 0], [9, 9], 16, 4, 9, 17, None, 4),                        # one token too many
    ([0, 2**31 - 1], [2**31 - 1, 2**31 - 1], 16, 4, 9, 17, 9, 7),   # lengths and counts past every limit
    ([3, 5], None, 16, 2, 4, 2, 5, 8),                              # a stack larger than the pool
    ([3, 5], None, 16, 2, 4, 2, -1, 8),
    ([1, -1, 1, 1], None, 16, 2, 9, 2, None, 4),                    # a token each, and room for two
    ([32, 1], None, 16, 2, 9, 2, None, 2),                          # a full row
    ([16] * 1100, None, 16, 2, 2199, 1100, None, 1),                # two workgroups
    ([0] * 50, [1000] * 50, 16, 63, 50 * 63 - 1, 50000, None, 1),   # refused by each of several workgroups
    ([2**31 - 1] * 4096, [2**31 - 1] * 4096, 256, 1, 1, 1, 1, 7),
])
def test_extend_refuses_on_the_gpu(lens, new, page, columns, pool, max_tokens, n_free, status, in_place):
    _run_extend(lens, new, page, columns, pool, max_tokens, in_place, status, n_free)


def test_extend_and_release_cycle():
    """Requests come and go: every page is in one row or on the stack, once."""
    page, columns, pool, n = 16, 6, 40, 9
    pages = rbs.Pages.allocate(n, columns, pool, page)
    table, free, n_free, lens = [[0] * columns for _ in range(n)], list(range(pool - 1, -1, -1)), pool, [-1] * n
    rng = torch.Generator().manual_seed(3)
    for k in range(60):
        admit = int(torch.randint(n, (1,), generator=rng))
        new = torch.randint(-1, 30, (n,), generator=rng).tolist()
        if lens[admit] < 0:
            lens[admit] = 0
            pages.seq_lens[admit] = 0
        step = rbs.rbs_pages_extend(pages, _ints(new), 120)
        want = R.extend(table, free, n_free, lens, new, page, 120)
        assert step.status.tolist() == [want["status"]]
        table, lens, n_free = want["table"], want["lens"], want["n_free"]
        assert pages.page_table.tolist() == table and pages.seq_lens.tolist() == lens
        assert step.slots.tolist() == want["slots"]
        out = [int(x) for x in (torch.rand(n, generator=rng) < 0.25)]
        status = rbs.rbs_pages_release(pages, _ints([x * 7 for x in out]))
        assert status.tolist() == [0]
        for row in range(n):
            if out[row] and lens[row] >= 0:
                for j in range(-(-lens[row] // page)):
                    free[n_free] = table[row][j]
                    n_free += 1
                lens[row] = -1
        assert pages.n_free.tolist() == [n_free] and pages.seq_lens.tolist() == lens
        assert pages.free_pages.tolist()[:n_free] == free[:n_free]
        owned = [table[r][j] for r in range(n) if lens[r] > 0 for j in range(-(-lens[r] // page))]
        assert sorted(owned + free[:n_free]) == list(range(pool))


@pytest.mark.parametrize("lens,n_free,pool,status", [
    ([40, 3], 2, 5, 8),       # three pages of row 0, one of row 1: more than the pool
    ([2**31 - 1, 3], 0, 5, 10),
    ([3, 3], 6, 5, 8),
    ([3, 3], -1, 5, 8),
])
def test_release_refuses_on_the_gpu(lens, n_free, pool, status):
    table, free = [[0, 1, 2], [3, -7, -7]], [4, 4, 4, 4, 4]
    pages = rbs.Pages(_ints(table), _ints(free), _ints([n_free]), _ints(lens), 16)
    assert rbs.rbs_pages_release(pages, _ints([1, 1])).tolist() == [status]
    assert pages.free_pages.tolist() == free and pages.n_free.tolist() == [n_free]
    assert pages.seq_lens.tolist() == lens and pages.page_table.tolist() == table


def test_release_of_many_rows():
    n, page, columns = 4096, 16, 5
    lens = [(13 * i) % 80 - 1 for i in range(n)]
    held = sum(-(-x // page) for x in lens if x > 0)
    table, free, n_free = _pages(lens, page, columns, held + 3, 8)
    pages = rbs.Pages(_ints(table), _ints(free), _ints([n_free]), _ints(lens), page)
    out = [i % 3 for i in range(n)]
    assert rbs.rbs_pages_release(pages, _ints(out)).tolist() == [0]
    for row in range(n):
        if out[row] and lens[row] >= 0:
            for j in range(-(-lens[row] // page)):
                free[n_free] = table[row][j]
                n_free += 1
            lens[row] = -1
    assert pages.seq_lens.tolist() == lens and pages.n_free.tolist() == [n_free]
    assert pages.free_pages.tolist() == free


# ------------------------------------------------------------------ norm and rotation

def _qkv(n, hq, hkv, seed, layout="qkv"):
    x = torch.randn(n, hq + 2 * hkv, D, generator=_gen(seed)) * 1.5
    x[:, :, ::17] *= 6.0
    x = x.to(torch.bfloat16)
    if layout == "qkv":
        b = x.cuda().transpose(0, 1)
        return b[:hq], b[hq:hq + hkv], b[hq + hkv:]
    parts = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])
    if layout == "heads":
        return tuple(p.transpose(0, 1).contiguous().cuda() for p in parts)
    return tuple(p.contiguous().cuda().transpose(0, 1) for p in parts)


def _cache(n_pages, hkv, page, fp8, layout="heads", amax=None, fill=0x5A):
    """A cache whose bytes are all `fill`, to see what was written."""
    if layout == "heads":
        shape, order = (n_pages, hkv, page, D), None
    else:
        shape, order = (n_pages, page, hkv, D), (1, 2)
    width = 1 if fp8 else 2
    bufs = [torch.full((*shape[:-1], D * width), fill, dtype=torch.uint8, device="cuda") for _ in range(2)]
    bufs = [b if fp8 else b.view(torch.bfloat16) for b in bufs]
    if order:
        bufs = [b.transpose(*order) for b in bufs]
    return rbs.PagedCache(*bufs, amax)


ROPE = [
    # tokens, heads, rot_dim, interleaved, norm, fp8 cache, page, layout of the inputs, of the cache, Q_out
    (1, 2, 1, 128, False, True, False, 16, "qkv", "heads", "new"),
    (1, 32, 4, 128, False, True, False, 16, "qkv", "heads", "in place"),
    (3, 7, 7, 128, True, True, True, 16, "heads", "tokens", "in place"),
    (5, 28, 4, 64, False, True, False, 32, "tokens", "tokens", "new"),
    (70, 64, 8, 32, True, True, True, 64, "qkv", "heads", "new"),
    (333, 5, 1, 8, False, True, False, 256, "qkv", "tokens", "in place"),
    (200, 6, 3, 0, False, True, True, 128, "heads", "heads", "new"),
    (41, 12, 2, 120, True, False, False, 16, "tokens", "heads", "in place"),
    (41, 12, 2, 120, False, False, True, 16, "qkv", "tokens", "new"),
    (4500, 9, 3, 96, False, True, False, 16, "qkv", "heads", "new"),
    (6, 512, 1, 128, False, True, False, 16, "tokens", "heads", "new"),
    (4111, 64, 8, 128, False, True, False, 16, "qkv", "heads", "in place"),   # 84 MB of rows: past the caches
    (4111, 64, 8, 96, True, True, True, 128, "qkv", "tokens", "new"),
    (4111, 64, 8, 72, False, True, False, 64, "tokens", "heads", "new"),       # (in runs of four)
]


@pytest.mark.parametrize("k", range(len(ROPE)))
def test_norm_rope(k):
    n, hq, hkv, rot, interleaved, norm, fp8, page, layout, cache_layout, out = ROPE[k]
    _say(f"[rope] {ROPE[k]}")
    g = _gen(20 + k)
    Q, K, V = _qkv(n, hq, hkv, 30 + k, layout)
    q0, k0, v0 = (x.cpu().double() for x in (Q, K, V))
    positions = torch.randint(0, 262144, (n,), generator=g, dtype=torch.int32)
    positions[0] = 2**31 - 1 if n > 1 else 131071
    pool = -(-n // page) + 2
    slots = torch.randperm(pool * page, generator=g)[:n].to(torch.int32)
    if n > 4:
        positions[3], positions[4] = -1, -2**31          # left out
        slots[1], slots[2] = -1, pool * page              # no place in the cache
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(torch.bfloat16) if norm else None for _ in range(2)]
    inv, factor = rbs.rope_frequencies(rot, scaling="parts", scale=4.0) if rot else (None, 1.0)
    rope = rbs.Rope(inv, *(None if x is None else x.cuda() for x in w), eps=1e-5, interleaved=interleaved, factor=factor)
    # Small magnitudes, so that some values saturate.
    amax = (torch.rand(2 * hkv, generator=g) * 4 + 0.5).cuda() if fp8 else None
    if fp8:
        amax[0] = 0.0
    cache = _cache(pool, hkv, page, fp8, cache_layout, amax)
    before = [x.contiguous().view(torch.uint8).cpu() for x in (cache.K, cache.V)]
    shape = rbs.make_shape(n, hq, hkv, 64)
    in_place = out == "in place"
    Qo, Ko = (Q, K) if in_place else (torch.full_like(Q, 7.0), torch.full_like(K, 7.0))
    got = rbs.rbs_qk_norm_rope(shape, rope, Q, K, positions.cuda(), V=V, cache=cache, slots=slots.cuda(), Q_out=Qo,
                               K_out=Ko)
    assert got[0] is Qo and got[1] is Ko
    left_out = positions < 0
    inv_c = None if inv is None else inv.cpu()
    for got, x0, weight in ((Qo, q0, w[0]), (Ko, k0, w[1])):
        y, size = R.norm_rope(x0, positions, inv_c, weight, 1e-5, interleaved, factor)
        a = got.cpu().double()
        kept = x0 if in_place else torch.full_like(x0, 7.0)
        assert torch.equal(a[:, left_out], kept[:, left_out])
        err, tol = (a - y).abs()[:, ~left_out], R.bf16_tolerance(y, size)[:, ~left_out]
        assert bool((err <= tol).all()), f"{(err / tol).max():.3f} of the tolerance"
    assert torch.equal(V.cpu().double(), v0)
    # The cache: the written slots, and every other byte as it was.
    y, size = R.norm_rope(k0, positions, inv_c, w[1], 1e-5, interleaved, factor)
    written = (~left_out) & (slots >= 0) & (slots < pool * page)
    at = slots[written].long()
    for i, (held, y, size) in enumerate(((cache.K, y, size), (cache.V, v0, v0.abs() * 0))):
        rows = held.cpu()[at // page, :, at % page].transpose(0, 1)
        y, size = y[:, written], size[:, written]
        if fp8:
            f = R.amax_factors(amax.cpu()[i * hkv:(i + 1) * hkv])[:, None, None]
            values = R.e4m3_values(rows)
            ys = (y * f).clamp(-448, 448)
            tol = R.code_tolerance(ys, size * f) + ys.abs() * 4 * R.U32
        else:
            values, ys, tol = rows.double(), y, R.bf16_tolerance(y, size)
            if i == 1:
                assert torch.equal(values, y)
        err = (values - ys).abs()
        assert bool((err <= tol).all()), f"cache {i}: {(err / tol).max():.3f} of the tolerance"
        after = held.contiguous().view(torch.uint8).cpu()
        same = torch.ones(pool * page, dtype=torch.bool)
        same[at] = False
        a, b = (z.transpose(1, 2).reshape(pool * page, -1)[same] for z in (after, before[i]))
        assert torch.equal(a, b), "places outside the slots were written"


def test_norm_rope_extreme_values():
    """Zeros, infinities and NaN stay in their own head rows."""
    n, hq, hkv = 9, 4, 2
    Q, K, V = _qkv(n, hq, hkv, 9)
    inv, _ = rbs.rope_frequencies()
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    rope = rbs.Rope(inv, w, w)
    shape = rbs.make_shape(n, hq, hkv, 64)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    clean = rbs.rbs_qk_norm_rope(shape, rope, Q, K, pos)
    Q[0, 1] = 0.0
    Q[1, 2, 5] = math.inf
    K[0, 3, 100] = math.nan
    V[1, 4, 3] = -math.inf
    V[0, 5, 7] = math.nan
    cache = _cache(1, hkv, 16, False)
    q, k = rbs.rbs_qk_norm_rope(shape, rope, Q, K, pos, V=V, cache=cache, slots=pos)
    assert bool((q[0, 1] == 0).all())
    assert bool(q[1, 2].isnan().any()) and bool(k[0, 3].isnan().all())
    other = torch.ones(hq, n, dtype=torch.bool, device="cuda")
    other[0, 1] = other[1, 2] = False
    assert torch.equal(q[other], clean[0][other])
    other = torch.ones(hkv, n, dtype=torch.bool, device="cuda")
    other[0, 3] = False
    assert torch.equal(k[other], clean[1][other])
    held = cache.V[0, :, :n]
    assert torch.equal(held.view(torch.int16), V.contiguous().view(torch.int16))


def test_norm_rope_without_a_cache():
    n, hq, hkv = 20, 4, 2
    Q, K, _ = _qkv(n, hq, hkv, 10)
    inv, _ = rbs.rope_frequencies(64)
    rope = rbs.Rope(inv, interleaved=True)
    shape, pos = rbs.make_shape(n, hq, hkv, 64), torch.arange(n, dtype=torch.int32, device="cuda")
    q, k = rbs.rbs_qk_norm_rope(shape, rope, Q, K, pos, keep_k=False)
    assert k is None
    y, size = R.norm_rope(Q.cpu().double(), pos.cpu(), inv.cpu(), None, 0.0, True, 1.0)
    assert bool(((q.cpu().double() - y).abs() <= R.bf16_tolerance(y, size)).all())


# ------------------------------------------------------------------ decode

def _decode_case(lens, hq, hkv, page, fp8, layout, seed, spare_columns=1, unused=math.nan, k_scale=1.0):
    """A cache filled for the lengths; every other place holds `unused`."""
    g = _gen(seed)
    n = len(lens)
    held = [-(-max(x, 0) // page) for x in lens]
    columns, pool = max(1, max(held)) + spare_columns, sum(held) + 2
    order = torch.randperm(pool, generator=g).tolist()
    table = torch.full((n, columns), -123456, dtype=torch.int32)
    live = torch.zeros(pool, page, dtype=torch.bool)
    for row, x in enumerate(lens):
        for j in range(held[row]):
            table[row, j] = order.pop()
            live[table[row, j], :min(page, x - j * page)] = True
    K = torch.randn(pool, hkv, page, D, generator=g) * k_scale + 0.3 * torch.randn(1, hkv, 1, D, generator=g)
    V = torch.randn(pool, hkv, page, D, generator=g) + 0.2
    q = (torch.randn(n, hq, D, generator=g) * 1.5).to(torch.bfloat16)
    amax = None
    if fp8:
        amax = torch.rand(2 * hkv, generator=g) * 3 + 2
        f = R.amax_factors(amax).float().view(2, 1, hkv, 1, 1)
        codes = [(x * y).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x, y in zip((K, V), f)]
        bad = 0x7F if math.isnan(unused) else 0x7E
        K, V = (torch.where(live[:, None, :, None], x, bad).to(torch.uint8) for x in codes)
    else:
        K, V = (torch.where(live[:, None, :, None], x.to(torch.bfloat16), torch.tensor(unused, dtype=torch.bfloat16))
                for x in (K, V))
    dev = [x.cuda() if layout == "heads" else x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (K, V)]
    cache = rbs.PagedCache(*dev, None if amax is None else amax.cuda())
    return dict(cache=cache, table=table, lens=lens, q=q, K=K, V=V, amax=amax, page=page, hq=hq, hkv=hkv, n=n)


def _values(c, which):
    if c["amax"] is None:
        return c[which].double()
    hkv = c["hkv"]
    a = c["amax"].double()[:hkv] if which == "K" else c["amax"].double()[hkv:]
    return R.e4m3_values(c[which]) * torch.where(a > 0, a / 448, torch.ones_like(a))[None, :, None, None]


def _check_decode(c, O, lse, scale, untouched=None):
    K, V = _values(c, "K"), _values(c, "V")
    worst = 0.0
    for row, n in enumerate(c["lens"]):
        if n < 0:
            continue
        k, v = (R.gather(x, c["table"][row], n, c["page"]) for x in (K, V))
        o, l, o_tol, l_tol = R.attend(c["q"][row].double(), k, v, scale)
        err = (O[:, row].cpu().double() - o).abs()
        assert bool((err <= o_tol).all()), f"row {row} of length {n}: {(err / (o_tol + 1e-300)).max():.3f} of the tolerance"
        if n > 0:
            worst = max(worst, float((err / o_tol).max()))
        if lse is not None:
            got = lse[:, row].cpu().double()
            if n == 0:
                assert bool((got == -math.inf).all())
            else:
                assert bool(((got - l).abs() <= l_tol).all()), f"row {row}: lse"
    return worst


def _run_decode(c, scale=0.0, q_layout="tokens", with_lse=True, ready=False, **more):
    q = c["q"].cuda()
    if q_layout == "tokens":
        Q = q.transpose(0, 1)
    elif q_layout == "heads":
        Q = q.transpose(0, 1).contiguous()
    else:  # a fused projection's view
        Q = torch.cat([q, torch.zeros(c["n"], 2 * c["hkv"], D, dtype=q.dtype, device="cuda")], 1).transpose(0, 1)[:c["hq"]]
    O = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device="cuda")
    O.fill_(math.nan)
    lse = torch.full((c["hq"], c["n"]), math.nan, device="cuda") if with_lse else None
    shape = rbs.make_shape(c["n"], c["hq"], c["hkv"], 64)
    table, lens = c["table"].cuda(), _ints(c["lens"])
    if ready:  # the call goes to another stream than the one that made its tensors
        torch.cuda.synchronize()
    got = rbs.rbs_paged_decode(shape, Q, c["cache"], table, lens, scale, O=O, lse=lse, **more)
    if ready:
        torch.cuda.synchronize()
    assert got is O
    return O, lse


DECODE = [
    # lengths, heads, page, fp8, cache layout, q layout, scale
    ([1], 2, 1, 16, False, "heads", "tokens", 0.0),
    ([0], 2, 1, 16, False, "heads", "heads", 0.0),
    ([0, 1, -1, 2, 15, 16, 17, 31, 32, 33, 0, -5], 8, 2, 16, False, "heads", "tokens", 0.0),
    ([0, 1, -1, 2, 15, 16, 17, 31, 32, 33, 0, -5], 8, 2, 16, True, "tokens", "tokens", 0.0),
    ([63, 64, 65, 127, 128, 129, 255, 256, 257, 500], 7, 1, 32, False, "tokens", "qkv", 0.3),
    ([63, 64, 65, 127, 128, 129, 255, 256, 257, 500], 7, 1, 64, True, "heads", "qkv", 0.05),
    ([1000, 3, 700], 5, 5, 128, False, "heads", "heads", 0.0),
    ([1000, 3, 700], 5, 5, 256, True, "tokens", "heads", 0.0),
    ([321, 40], 16, 1, 16, False, "heads", "tokens", 0.0),
    ([321, 40], 34, 2, 16, False, "tokens", "tokens", 0.0),      # 17 heads to a KV head
    ([321, 40, 0], 33, 1, 32, True, "heads", "tokens", 0.0),
    ([77, 0, 2000], 512, 4, 64, False, "heads", "tokens", 0.0),  # 128 heads to a KV head
    ([40] * 300, 4, 2, 16, False, "heads", "tokens", 0.0),
    ([(i * 37) % 90 - 1 for i in range(1500)], 2, 1, 16, True, "heads", "tokens", 0.0),
    ([9000, 2, 4097, 0, 12345], 8, 2, 16, False, "heads", "tokens", 0.0),
    ([9000, 2, 4097, 0, 12345], 8, 2, 128, True, "heads", "tokens", 0.0),
    ([65537], 4, 4, 256, False, "tokens", "tokens", 0.0),
    ([(i * 53) % 260 for i in range(700)], 16, 8, 16, False, "heads", "tokens", 0.0),    # a wave to a row
    ([(i * 53) % 500 - 1 for i in range(700)], 14, 2, 32, True, "heads", "qkv", 0.0),
    ([(i * 53) % 90 for i in range(600)] + [1500], 8, 8, 64, False, "tokens", "tokens", 0.0),  # and one long row
    ([150] * 520 + [2500] * 3, 16, 1, 16, False, "heads", "tokens", 0.0),                # more rows than workers
    ([384, 383, 1] * 5, 8, 2, 32, False, "heads", "tokens", 0.0),                         # one launch up to here
    ([385, 383, 1] * 5, 8, 2, 16, False, "heads", "tokens", 0.0),
    ([768, 700, 0] * 5, 8, 2, 16, True, "heads", "tokens", 0.0),
    ([768] * 3, 8, 1, 256, False, "heads", "tokens", 0.0),
    ([769, 1, 768], 8, 1, 16, False, "heads", "tokens", 0.0),
    ([4000] * 70 + [1], 8, 2, 64, True, "heads", "tokens", 0.0),                          # past the caches
    ([5000] * 8 + [0, 33], 16, 4, 16, False, "tokens", "tokens", 0.0),
    ([70] + [0] * 2000 + [-1] * 2000 + [3000, 33], 8, 2, 16, False, "heads", "tokens", 0.0),  # few rows used
    ([0] * 50 + [20] * 3 + [-1] * 900 + [40] * 2, 4, 1, 32, True, "heads", "tokens", 0.0),
    ([512, 3000], 512, 512, 16, False, "heads", "tokens", 0.0),                           # as many units as workers
    ([150001], 8, 1, 64, False, "heads", "tokens", 0.0),
]


@pytest.mark.parametrize("k", range(len(DECODE)))
def test_decode(k):
    lens, hq, hkv, page, fp8, layout, q_layout, scale = DECODE[k]
    _say(f"[decode] {len(lens)} rows, heads {hq}/{hkv}, page {page}, fp8 {fp8}")
    c = _decode_case(lens, hq, hkv, page, fp8, layout, 50 + k)
    O, lse = _run_decode(c, scale, q_layout)
    worst = _check_decode(c, O, lse, scale if scale > 0 else 1 / math.sqrt(D))
    _say(f"[decode] {worst:.3f} of the tolerance")
    unused = [row for row, n in enumerate(lens) if n < 0]
    assert bool(O[:, unused].isnan().all()) and bool(lse[:, unused].isnan().all())
    O2, _ = _run_decode(c, scale, q_layout, with_lse=False)
    assert torch.equal(O.nan_to_num(9.0), O2.nan_to_num(9.0)), "the same call again"


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_large_logits(fp8):
    """Logits of some hundreds: one key takes nearly all, and the running maximum jumps by many powers."""
    lens = [700, 33, 5000]
    c = _decode_case(lens, 8, 2, 16, fp8, "heads", 91, k_scale=12.0)
    O, lse = _run_decode(c, 2.0)
    _check_decode(c, O, lse, 2.0)


def test_decode_infinities_past_the_length():
    c = _decode_case([17, 100, 4], 4, 2, 64, False, "heads", 92, unused=math.inf)
    O, lse = _run_decode(c)
    _check_decode(c, O, lse, 1 / math.sqrt(D))


def test_decode_clamps_lengths_and_pages():
    """Lengths past the table and page numbers outside the cache stay inside the buffers."""
    c = _decode_case([64, 64], 4, 2, 16, False, "heads", 93, spare_columns=0, unused=0.0)
    want, _ = _run_decode(c)
    long = dict(c, lens=[2**31 - 1, 64])
    got, _ = _run_decode(long)
    assert torch.equal(got, want)
    pool = c["K"].shape[0]
    wild = dict(c, table=c["table"].clone())
    wild["table"][0, 1], wild["table"][0, 2] = 2**31 - 1, -2**31
    tame = dict(c, table=c["table"].clone())
    tame["table"][0, 1], tame["table"][0, 2] = pool - 1, 0
    assert torch.equal(_run_decode(wild)[0].nan_to_num(3.0), _run_decode(tame)[0].nan_to_num(3.0))


def test_decode_pages_past_32_bits():
    """A cache of more than 2^32 bytes (and 2^31 elements) a tensor: the same rows in its first and last pages."""
    page, hkv, hq = 256, 8, 16
    n_pages = (1 << 31) // (page * hkv * D) + 40
    c = _decode_case([5000, 300], hq, hkv, page, False, "heads", 94, unused=0.0)
    small = c["K"].shape[0]
    K = torch.empty(n_pages, hkv, page, D, dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    K[-small:], V[-small:] = c["K"].cuda(), c["V"].cuda()
    far = dict(c, cache=rbs.PagedCache(K, V), table=torch.where(c["table"] >= 0, c["table"] + n_pages - small, c["table"]))
    want, got = _run_decode(c), _run_decode(far)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # and written there by the norm and rotation call
    Q, Kn, Vn = _qkv(4, hq, hkv, 95)
    slots = _ints([(n_pages - 1) * page + 255, (n_pages - 3) * page, 7, -1])
    rbs.rbs_qk_norm_rope(rbs.make_shape(4, hq, hkv, 64), rbs.Rope(None), Q, Kn, _ints([1, 2, 3, 4]), V=Vn,
                         cache=far["cache"], slots=slots)
    assert torch.equal(K[-1, :, 255], Kn[:, 0]) and torch.equal(V[-3, :, 0], Vn[:, 1]) and torch.equal(V[0, :, 7], Vn[:, 2])


@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_keys_and_values_in_one_buffer(order):
    """[n_pages][2][..]: written by the norm and rotation call, read by the attention."""
    n, hq, hkv, page, pool = 40, 8, 2, 16, 7
    inner = (hkv, page) if order == "heads" else (page, hkv)
    both = torch.full((pool, 2, *inner, D), math.nan, dtype=torch.bfloat16, device="cuda")
    K, V = (both[:, i] if order == "heads" else both[:, i].transpose(1, 2) for i in range(2))
    cache = rbs.PagedCache(K, V)
    Q, Kn, Vn = _qkv(n, hq, hkv, 31)
    table = torch.tensor([[5, 0, 3]], dtype=torch.int32)
    at = torch.arange(n)
    slots = (table[0, at // page] * page + at % page).to(torch.int32)
    shape = rbs.make_shape(n, hq, hkv, 64)
    q, k = rbs.rbs_qk_norm_rope(shape, rbs.Rope(rbs.rope_frequencies()[0]), Q, Kn, at.to(torch.int32).cuda(), V=Vn,
                                cache=cache, slots=slots.cuda())
    last = q[:, -1:]
    lse = torch.empty(hq, 1, device="cuda")
    O = rbs.rbs_paged_decode(rbs.make_shape(1, hq, hkv, 64), last, cache, table.cuda(), _ints([n]), lse=lse)
    o, l, o_tol, l_tol = R.attend(last[:, 0].cpu().double(), k.cpu().double(), Vn.cpu().double(), 1 / math.sqrt(D))
    assert bool(((O[:, 0].cpu().double() - o).abs() <= o_tol).all())
    assert bool(((lse[:, 0].cpu().double() - l).abs() <= l_tol).all())
    assert bool(both[[1, 2, 4, 6]].isnan().all())


def test_decode_with_heads_of_scale_one():
    """amax 0: the codes stand for themselves."""
    c = _decode_case([300, 40], 4, 2, 16, True, "heads", 99)
    c["amax"][0] = c["amax"][3] = 0.0
    c["cache"].amax.copy_(c["amax"])
    O, lse = _run_decode(c, 0.01)
    _check_decode(c, O, lse, 0.01)


def test_decode_on_a_side_stream_and_own_workspace():
    c = _decode_case([3000, 77, 4096], 8, 2, 32, False, "heads", 96)
    want = _run_decode(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = _run_decode(c)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s.wait_stream(torch.cuda.current_stream())
    got = _run_decode(c, stream=s, ready=True)  # given by name, from another current stream
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with torch.cuda.stream(s):
        got = _run_decode(c, stream=torch.cuda.default_stream(), ready=True)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws = torch.full((rbs.rbs_decode_workspace_bytes() // 4,), math.nan, device="cuda")
    for _ in range(2):  # whatever the workspace holds, also after a larger call
        got = _run_decode(c, workspace=ws)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        ws.view(torch.int32).fill_(0x7FFFFFFF)
    small = _decode_case([5, 300], 8, 2, 32, False, "heads", 97)
    _check_decode(small, *_run_decode(small, workspace=ws), 1 / math.sqrt(D))


def test_outputs_are_written_and_nothing_past_them():
    c = _decode_case([300, 0, 20], 8, 2, 32, False, "heads", 98)
    n = 8 * 3 * D
    full = torch.full((n + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    lfull = torch.full((24 + 64,), 7.0, device="cuda")
    Q = c["q"].cuda().transpose(0, 1).contiguous()
    ws = torch.full((rbs.rbs_decode_workspace_bytes() // 4 + 64,), 3.0, device="cuda")
    rbs.rbs_paged_decode(rbs.make_shape(3, 8, 2, 64), Q, c["cache"], c["table"].cuda(), _ints(c["lens"]),
                         O=full[:n].view(8, 3, D), lse=lfull[:24].view(8, 3), workspace=ws)
    _check_decode(c, full[:n].view(8, 3, D), lfull[:24].view(8, 3), 1 / math.sqrt(D))
    assert bool((full[n:] == 7).all()) and bool((lfull[24:] == 7).all()) and bool((ws[-64:] == 3).all())


# ------------------------------------------------------------------ together

def _layer(seed, hq, hkv, rot=128, fp8_amax=None):
    g = _gen(seed)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16) for _ in range(2)]
    inv, factor = rbs.rope_frequencies(rot)
    return rbs.Rope(inv, w[0].cuda(), w[1].cuda(), factor=factor), w, inv.cpu()


@pytest.mark.parametrize("fp8", [False, True])
def test_prompts_then_decode_steps(fp8):
    """Two prompts through the sparse prefill's dense lists, then six decode steps with a request admitted and
    one released on the way; every step against 64-bit attention over all of a request's tokens."""
    hq, hkv, page, rows = 8, 2, 16, 4
    rope, w, inv = _layer(7, hq, hkv)
    amax = torch.full((2 * hkv,), 7.0).cuda() if fp8 else None
    cache = _cache(40, hkv, page, fp8, "heads", amax, fill=0xFF)  # NaN everywhere
    pages = rbs.Pages.allocate(rows, 12, 40, page)
    known = {r: [torch.zeros(hkv, 0, D, dtype=torch.float64) for _ in range(2)] for r in range(rows)}  # as held
    scale = 1 / math.sqrt(D)

    def project(n, seed):
        Q, K, V = _qkv(n, hq, hkv, seed)
        return Q, K, V

    def remember(step, n, rows_of):
        """What the cache holds of the new tokens (its values were checked by the tests above)."""
        slots = step.slots.tolist()
        for t in range(n):
            p, at = slots[t] // page, slots[t] % page
            for i, x in enumerate((cache.K, cache.V)):
                v = x[p, :, at].cpu()
                v = R.e4m3_values(v) * 7.0 / 448 if fp8 else v.double()
                known[rows_of[t]][i] = torch.cat([known[rows_of[t]][i], v[:, None]], 1)

    # Prompts of 70 and 33 tokens in rows 0 and 2.
    prompt = [70, 0, 33, 0]
    pages.seq_lens[0] = 0
    pages.seq_lens[2] = 0
    step = rbs.rbs_pages_extend(pages, _ints(prompt), 110)
    assert step.status.tolist() == [0] and step.cu_tokens.tolist() == [0, 70, 70, 103, 103]
    Q, K, V = project(110, 1)
    batch = rbs.Batch([70, 33])
    shape = rbs.varlen_shape(batch, hq, hkv, 64)
    rbs.rbs_qk_norm_rope(rbs.make_shape(110, hq, hkv, 64), rope, Q, K, step.positions, V=V, cache=cache,
                         slots=step.slots, Q_out=Q, K_out=K)
    remember(step, 103, [0] * 70 + [2] * 33)
    Qp, Kp, Vp = Q[:, :103], K[:, :103], V[:, :103]
    counts, indices = rbs.rbs_dense_indices_varlen(shape, batch)
    O = rbs.rbs_sparse_prefill_varlen(shape, batch, Qp, Kp, Vp, counts, indices)
    last = Qp[:, 69].cpu().double()
    k70, v70 = (x[:, :70].cpu().double() for x in (Kp, Vp))
    o, _, o_tol, _ = R.attend(last, k70, v70, scale)
    size = R.attend(last, k70, v70.abs(), scale)[0]
    # The prefill holds its weights in bf16: each is off by at most half a step, which moves the weighted values by
    # HALF_BF16 of their absolute sum and the denominator by HALF_BF16 of itself; then o_tol (fp32 and the last rounding).
    assert bool(((O[:, 69].cpu().double() - o).abs() <= o_tol + R.HALF_BF16 * (size + o.abs()) * 1.01).all())
    for k in range(6):
        if k == 2:
            pages.seq_lens[3] = 0  # a request that starts from nothing
        if k == 4:
            assert rbs.rbs_pages_release(pages, _ints([0, 0, 1, 0])).tolist() == [0]
            known[2] = [x[:, :0] for x in known[2]]
        step = rbs.rbs_pages_extend(pages, None, rows)
        cu = step.cu_tokens.tolist()
        lens = step.seq_lens.tolist()
        rows_of = [r for r in range(rows) for _ in range(cu[r + 1] - cu[r])]
        n = cu[rows]
        assert step.status.tolist() == [0] and n == (2, 2, 3, 3, 2, 2)[k]
        Qn, Kn, Vn = project(rows, 100 + k)
        q, _ = rbs.rbs_qk_norm_rope(rbs.make_shape(rows, hq, hkv, 64), rope, Qn, Kn, step.positions, V=Vn, cache=cache,
                                    slots=step.slots, keep_k=False)
        remember(step, n, rows_of)
        # The used rows' queries at their rows of the table.
        Qr = torch.zeros(rows, hq, D, dtype=torch.bfloat16, device="cuda")
        Qr[rows_of] = q[:, :n].transpose(0, 1)
        lse = torch.empty(hq, rows, device="cuda")
        O = rbs.rbs_paged_decode(rbs.make_shape(rows, hq, hkv, 64), Qr.transpose(0, 1), cache, pages.page_table,
                                 step.seq_lens, lse=lse)
        for r in range(rows):
            if lens[r] < 0:
                continue
            kk, vv = known[r]
            assert kk.shape[1] == lens[r]
            o, l, o_tol, l_tol = R.attend(Qr[r].cpu().double(), kk, vv, scale)
            assert bool(((O[:, r].cpu().double() - o).abs() <= o_tol).all())
            assert bool(((lse[:, r].cpu().double() - l).abs() <= l_tol).all())


def test_captured_steps_side_by_side():
    """Two decode steps captured into graphs on one stream, replayed three times each (also at once, on two
    streams) with eager calls in between: every replay equals the eager step from the same state."""
    hq, hkv, page, rows = 8, 2, 16, 5
    rope, _, _ = _layer(8, hq, hkv)
    shape = rbs.make_shape(rows, hq, hkv, 64)

    class Server:
        def __init__(self, seed):
            g = _gen(seed)
            self.lens0 = [int(x) for x in torch.randint(0, 5000, (rows,), generator=g)]
            held = [-(-x // page) for x in self.lens0]
            pool = sum(held) + 3 * rows
            table, free, n_free = _pages(self.lens0, page, max(held) + 2, pool, seed)
            self.pages = rbs.Pages(_ints(table).clamp(min=0), _ints(free), _ints([n_free]), _ints(self.lens0), page)
            self.cache = rbs.PagedCache.allocate(pool, page, hkv)
            self.cache.K.normal_()
            self.cache.V.normal_()
            self.n_free0 = n_free
            self.Q, self.K, self.V = _qkv(rows, hq, hkv, seed + 1)
            self.out = rbs.PageStep.allocate(self.pages, rows)
            self.table0, self.K0 = self.pages.page_table.clone(), self.cache.K.clone()

        def reset(self):
            self.pages.seq_lens.copy_(_ints(self.lens0))
            self.pages.n_free.fill_(self.n_free0)
            self.pages.page_table.copy_(self.table0)
            self.cache.K.copy_(self.K0)

        def step(self):
            o = rbs.rbs_pages_extend(self.pages, step=self.out)
            q, _ = rbs.rbs_qk_norm_rope(shape, rope, self.Q, self.K, o.positions, V=self.V, cache=self.cache,
                                        slots=o.slots, keep_k=False)
            return rbs.rbs_paged_decode(shape, q, self.cache, self.pages.page_table, o.seq_lens)

    servers = [Server(200), Server(300)]
    want = []
    for v in servers:
        steps = []
        v.reset()
        for _ in range(3):
            steps.append(v.step().clone())
        want.append(steps)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for v in servers:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(v.step())
        graphs.append(g)
    for v in servers:
        v.reset()
    other = torch.cuda.Stream()
    for k in range(3):
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], want[i][k]), f"replay {k} of graph {i}"
            assert servers[i].pages.seq_lens.tolist() == [x + k + 1 for x in servers[i].lens0]
        c = _decode_case([3000, 5], hq, hkv, page, False, "heads", 400 + k)
        _check_decode(c, *_run_decode(c), 1 / math.sqrt(D))


# ------------------------------------------------------------------ threads

def test_threads_that_decode_on_one_stream():
    """Rows in parts (two launches a call), calls of three threads between each other."""
    import threading
    cases = [_decode_case(lens, 8, 2, 16, False, "heads", 500 + k)
             for k, lens in enumerate(([3000, 900, 0, 2100], [4000], [1500] * 30))]
    want = [_run_decode(c) for c in cases]
    held = [(c["q"].cuda().transpose(0, 1), c["table"].cuda(), _ints(c["lens"])) for c in cases]
    torch.cuda.synchronize()
    got, failed, start = [[] for _ in cases], [], threading.Barrier(len(cases))

    def calls(k):
        try:
            c, (Q, table, lens) = cases[k], held[k]
            shape = rbs.make_shape(c["n"], c["hq"], c["hkv"], 64)
            start.wait()
            for _ in range(60):
                lse = torch.empty(c["hq"], c["n"], device="cuda")
                got[k].append((rbs.rbs_paged_decode(shape, Q, c["cache"], table, lens, lse=lse), lse))
        except Exception as e:  # (shown below: a thread's own traceback is not the test's)
            failed.append(e)

    threads = [threading.Thread(target=calls, args=(k,)) for k in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for k, (o, l) in enumerate(want):
        assert len(got[k]) == 60
        for O, lse in got[k]:
            assert torch.equal(O, o) and torch.equal(lse, l)


# ------------------------------------------------------------------ queries packed row after row

def _run_packed(c, new, behind, scale=0.0, cu=None):
    """Random queries for every token of a batch in which row s has new[s] (unused rows: none); O and lse, the
    token of each row that has one, and those queries."""
    add = [max(0, a) if n >= 0 else 0 for n, a in zip(c["lens"], new)]
    at = [0]
    for a in add:
        at.append(at[-1] + a)
    n = max(1, at[-1] + behind)
    Q = (torch.randn(n, c["hq"], D, generator=_gen(len(c["lens"]) + n)) * 1.5).to(torch.bfloat16)
    Qd = Q.cuda().transpose(0, 1)
    O = torch.full_like(Qd, math.nan)
    lse = torch.full((c["hq"], n), math.nan, device="cuda")
    got = rbs.rbs_paged_decode(rbs.make_shape(n, c["hq"], c["hkv"], 64), Qd, c["cache"], c["table"].cuda(),
                               _ints(c["lens"]), scale, O=O, lse=lse, cu_tokens=_ints(at if cu is None else cu))
    assert got is O
    return O, lse, {row: at[row + 1] - 1 for row, a in enumerate(add) if a > 0}, Q


def _check_packed(c, O, lse, token, Q, scale):
    K, V = _values(c, "K"), _values(c, "V")
    for row, t in token.items():
        n = c["lens"][row]
        k, v = (R.gather(x, c["table"][row], n, c["page"]) for x in (K, V))
        o, l, o_tol, l_tol = R.attend(Q[t].double(), k, v, scale)
        assert bool(((O[:, t].cpu().double() - o).abs() <= o_tol).all()), f"row {row} of length {n}, token {t}"
        got = lse[:, t].cpu().double()
        assert bool(((got - l).abs() <= l_tol).all()) if n > 0 else bool((got == -math.inf).all())
    others = [t for t in range(O.shape[1]) if t not in token.values()]
    assert bool(O[:, others].isnan().all()) and bool(lse[:, others].isnan().all()), "other tokens were written"


PACKED = [
    # lengths, new tokens, tokens behind the last, heads, page, fp8, columns to spare
    ([-1, 5], [1, 1], 0, 2, 1, 16, False, 1),
    ([-1, -1], [1, 1], 3, 2, 1, 16, False, 1),                                    # no token at all
    ([70, -1, 33, 0, -1, 200], [1] * 6, 2, 8, 2, 16, False, 0),                    # one launch
    ([70, -1, 33, 0, -1, 200], [1] * 6, 2, 8, 2, 16, True, 0),
    ([3000, -1, 900, 40, -1, 5000, 17], [1, 1, 0, 1, 1, 1, 1], 1, 28, 4, 16, False, 60),   # rows in parts, one with none
    ([3000, -1, 900, 40, -1, 5000, 17], [3, 1, 0, 800, 1, 1, 17], 5, 28, 4, 32, True, 0),   # a last token each
    ([-1, 9000, -1], [1, 1, 1], 0, 8, 1, 64, False, 300),                                   # a wide table
    ([(i * 53) % 90 - 1 for i in range(700)], [1 - (i % 7 == 3) for i in range(700)], 9, 16, 8, 16, False, 0),
    ([(i * 53) % 1500 - 1 if i % 4 else -1 for i in range(300)], [1] * 300, 75, 8, 2, 32, True, 0),
    ([(i * 53) % 700 - 1 if i % 3 else -1 for i in range(90)], [1] * 90, 0, 64, 32, 16, False, 0),   # fewer workers than rows
    ([2000, -1, 10], [1, 1, 1], 0, 34, 2, 16, False, 0),                                    # 17 heads to a KV head
    ([-1] * 3000 + [600, 2], [1] * 3002, 40, 4, 2, 16, False, 0),
]


@pytest.mark.parametrize("k", range(len(PACKED)))
def test_decode_of_packed_queries(k):
    lens, new, behind, hq, hkv, page, fp8, spare = PACKED[k]
    _say(f"[packed] {len(lens)} rows, heads {hq}/{hkv}, page {page}, fp8 {fp8}")
    c = _decode_case(lens, hq, hkv, page, fp8, "heads", 600 + k, spare_columns=spare)
    _check_packed(c, *_run_packed(c, new, behind, 0.1), 0.1)


def test_packed_queries_with_a_row_each_are_those_by_row():
    """Every row used: token t is row t's, and the two forms give the same bits."""
    c = _decode_case([300, 4000, 1, 77, 2500], 8, 2, 16, False, "heads", 640)
    O, lse = _run_decode(c)
    Q = c["q"].cuda().transpose(0, 1)
    l2 = torch.empty_like(lse)
    O2 = rbs.rbs_paged_decode(rbs.make_shape(5, 8, 2, 64), Q, c["cache"], c["table"].cuda(), _ints(c["lens"]), lse=l2,
                              cu_tokens=_ints([0, 1, 2, 3, 4, 5]))
    assert torch.equal(O2, O) and torch.equal(l2, lse)


def test_packed_offsets_outside_the_tokens():
    """Rows whose offsets fall outside the queries have no token; nothing is read or written there."""
    c = _decode_case([3000, 40, 500, 20, 900], 8, 2, 16, False, "heads", 641)
    cu = [-5, 0, 1, 2**31 - 1, -2**31, 2]   # rows 1 and 4 have tokens 0 and 1 of three
    O, lse, _, Q = _run_packed(c, [1, 1, 1, 0, 0], 0, cu=cu)
    _check_packed(c, O, lse, {1: 0, 4: 1}, Q, 1 / math.sqrt(D))


@pytest.mark.parametrize("fp8", [False, True])
def test_steps_with_unused_rows(fp8):
    """The three calls chained with rows unused, admitted and released between them, before used ones too: nothing is
    read back for the next call, and captured steps equal the eager ones."""
    hq, hkv, page, rows, steps = 8, 2, 16, 6, 7
    rope, _, _ = _layer(9, hq, hkv)
    amax = torch.full((2 * hkv,), 7.0).cuda() if fp8 else None
    shape = rbs.make_shape(rows, hq, hkv, 64)
    inputs = [_qkv(rows, hq, hkv, 700 + k) for k in range(steps)]
    now = [torch.empty_like(x) for x in inputs[0]]  # what the graph reads

    class Server:
        def __init__(self):
            self.pages = rbs.Pages.allocate(rows, 400, 500, page)
            self.cache = _cache(500, hkv, page, fp8, "heads", amax, fill=0xFF)  # NaN everywhere
            self.out = rbs.PageStep.allocate(self.pages, rows)
            self.O = torch.full((rows, hq, D), math.nan, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
            self.lse = torch.full((hq, rows), math.nan, device="cuda")
            for row, n in ((1, 1000), (3, 40)):  # prompts in rows 1 and 3; rows 0, 2, 4 and 5 unused
                self.pages.seq_lens[row] = 0
                Q, K, V = _qkv(n, hq, hkv, 720 + row)
                counts = torch.zeros(rows, dtype=torch.int32, device="cuda")
                counts[row] = n
                s = rbs.rbs_pages_extend(self.pages, counts, n)
                rbs.rbs_qk_norm_rope(rbs.make_shape(n, hq, hkv, 64), rope, Q, K, s.positions, V=V, cache=self.cache,
                                     slots=s.slots, keep_k=False)

        def between(self, k):
            if k == 2:
                self.pages.seq_lens[5] = 0
            if k == 3:
                self.pages.seq_lens[0] = 0
            if k == 5:
                rbs.rbs_pages_release(self.pages, _ints([0, 1, 0, 0, 0, 0]))

        def step(self):
            Q, K, V = now
            o = rbs.rbs_pages_extend(self.pages, step=self.out)
            self.q, _ = rbs.rbs_qk_norm_rope(shape, rope, Q, K, o.positions, V=V, cache=self.cache, slots=o.slots,
                                             keep_k=False)
            return rbs.rbs_paged_decode(shape, self.q, self.cache, self.pages.page_table, o.seq_lens, O=self.O,
                                        lse=self.lse, cu_tokens=o.cu_tokens)

    eager, want = Server(), []
    used_at = [[1, 3], [1, 3], [1, 3, 5], [0, 1, 3, 5], [0, 1, 3, 5], [0, 3, 5], [0, 3, 5]]
    for k in range(steps):
        eager.between(k)
        for a, b in zip(now, inputs[k]):
            a.copy_(b)
        eager.step()
        lens, used = eager.pages.seq_lens.tolist(), used_at[k]
        assert [r for r in range(rows) if lens[r] >= 0] == used and eager.out.status.tolist() == [0]
        table, (kc, vc) = eager.pages.page_table.cpu(), (x.cpu() for x in (eager.cache.K, eager.cache.V))
        for t, row in enumerate(used):
            held = [R.gather(x, table[row], lens[row], page) for x in (kc, vc)]
            held = [R.e4m3_values(x) * 7.0 / 448 if fp8 else x.double() for x in held]
            o, l, o_tol, l_tol = R.attend(eager.q[:, t].cpu().double(), *held, 1 / math.sqrt(D))
            assert bool(((eager.O[:, t].cpu().double() - o).abs() <= o_tol).all()), f"step {k}, row {row}"
            assert bool(((eager.lse[:, t].cpu().double() - l).abs() <= l_tol).all())
        want.append((eager.O.clone(), eager.lse.clone()))
    captured = Server()
    for a, b in zip(now, inputs[0]):
        a.copy_(b)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        captured.step()
    for k in range(steps):
        captured.between(k)
        for a, b in zip(now, inputs[k]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        n = len(used_at[k])
        assert torch.equal(captured.O[:, :n], want[k][0][:, :n]) and torch.equal(captured.lse[:, :n], want[k][1][:, :n])


# ------------------------------------------------------------------ streams given by name

def _memory_of(t):
    """Handle of the stream whose memory a tensor is."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not torch's memory")


@pytest.mark.parametrize("which", ["side", "default", "current"])
def test_outputs_are_the_memory_of_the_calls_stream(which):
    """What a call on a stream given by name makes itself: memory of another stream may still be in use there."""
    hq, hkv, page, rows = 8, 2, 16, 3
    side = torch.cuda.Stream()
    stream = dict(side=side, default=torch.cuda.default_stream(), current=None)[which]
    here = side if which == "default" else torch.cuda.default_stream()
    handle = here.cuda_stream if stream is None else stream.cuda_stream
    c = _decode_case([300, 40, 2000], hq, hkv, page, False, "heads", 650)
    shape, rope = rbs.make_shape(rows, hq, hkv, 64), rbs.Rope(rbs.rope_frequencies()[0])
    pages = rbs.Pages.allocate(rows, 9, 20, page)
    pages.seq_lens.zero_()
    Q, K, V = _qkv(rows, hq, hkv, 651)
    cache, lens, table = _cache(20, hkv, page, False), _ints(c["lens"]), c["table"].cuda()
    released = _ints([1, 0, 1])
    queries = c["q"].cuda().transpose(0, 1)
    torch.cuda.synchronize()
    with torch.cuda.stream(here):
        step = rbs.rbs_pages_extend(pages, stream=stream)
        q, k = rbs.rbs_qk_norm_rope(shape, rope, Q, K, step.positions, V=V, cache=cache, slots=step.slots, stream=stream)
        O = rbs.rbs_paged_decode(shape, queries, c["cache"], table, lens, stream=stream)
        status = rbs.rbs_pages_release(pages, released, stream=stream)
    torch.cuda.synchronize()
    for t in (step.cu_tokens, step.positions, step.slots, step.status, q, k, O, status):
        assert _memory_of(t) == handle
    assert step.seq_lens is pages.seq_lens and pages.seq_lens.tolist() == [-1, 1, -1] and status.tolist() == [0]
    assert torch.equal(cache.K[:3, :, 0].transpose(0, 1), k[:, :])
    _check_decode(c, O, None, 1 / math.sqrt(D))


@pytest.mark.parametrize("n,hkv", [(1, 2), (5, 1)])
def test_values_of_another_layout(n, hkv):
    """One token, or one KV head: V's stride over it is not K's, and not used."""
    hq, page = 4, 16
    Q, K, V = _qkv(n, hq, hkv, 660, "heads")
    far = torch.zeros(hkv + 2, n + 3, D, dtype=torch.bfloat16, device="cuda")
    V2 = far[:hkv, :n] if n == 1 else far[:hkv].as_strided((1, n, D), (9 * far.stride(0), D, 1))
    V2.copy_(V)
    if n == 1:  # (head, token, dimension) of a buffer whose tokens are far apart
        V2 = V2.transpose(0, 1).contiguous().transpose(0, 1)
        K = K.as_strided((hkv, 1, D), (D, D, 1))
    assert V2.stride() != K.stride()
    cache, slots = _cache(2, hkv, page, False), torch.arange(n, dtype=torch.int32, device="cuda") + 3
    rbs.rbs_qk_norm_rope(rbs.make_shape(n, hq, hkv, 64), rbs.Rope(None), Q, K, slots, V=V2, cache=cache, slots=slots)
    assert torch.equal(cache.V[0, :, 3:3 + n], V) and torch.equal(cache.K[0, :, 3:3 + n], K)


# ------------------------------------------------------------------ every key once

LONG = [
    # lengths, heads, page, fp8, with the log-sum-exp of the longest row known to a key
    ([150001], 8, 1, 64, False),                          # parts of 512 workers, joined by single columns
    ([150001], 8, 1, 64, True),
    ([150001] + [700] * 30, 32, 4, 16, False),             # four columns a join
    ([150001] + [700] * 30, 32, 4, 32, True),
    ([700] * 9 + [40000] + [5] * 10, 64, 32, 128, False),  # fewer workers than rows: a record for each worker
    ([700] * 9 + [40000] + [5] * 10, 64, 32, 128, True),
    ([50000, 33, 49999], 34, 2, 256, False),               # 17 heads to a KV head
]


@pytest.mark.parametrize("k", range(len(LONG)))
def test_every_key_counts_once(k):
    """Keys of 0, so that every weight is 1: the log-sum-exp is ln n, to less than one key more or less would make,
    and values that mark their tile of 32 (FP8: 64) keys in one element each, so that a tile (a part) that is lost or
    counted twice shows in that element.

    Sums of ones and of marks are whole numbers below 2^24, exact in fp32 in any order.  lse = log2(n) ln 2: the
    logarithm to 2 of its steps (2^-19 each from 16 on), the product and its constant to half a step each: 4.1e-6
    for 150001 keys (one key: 6.7e-6).  O = count / n: a division, a product and bf16, half a step of bf16 and 4 of
    fp32."""
    lens, hq, hkv, page, fp8 = LONG[k]
    _say(f"[once] {len(lens)} rows, heads {hq}/{hkv}, page {page}, fp8 {fp8}")
    tile, n = 64 if fp8 else 32, len(lens)
    held = [-(-x // page) for x in lens]
    pool = sum(held)
    order = torch.randperm(pool, generator=_gen(670 + k)).to(torch.int32)
    table = torch.full((n, max(held) + 1), -1, dtype=torch.int32)
    at = 0
    for row, h in enumerate(held):
        table[row, :h] = order[at:at + h]
        at += h
    one = 0x38 if fp8 else 1.0
    kind = torch.uint8 if fp8 else torch.bfloat16
    K = torch.zeros(pool, hkv, page, D, dtype=kind, device="cuda")
    V = torch.zeros_like(K)
    want = torch.zeros(n, D, dtype=torch.float64)
    for row, x in enumerate(lens):
        j = torch.arange(x)
        mark = (j // tile) % D
        want[row] = torch.bincount(mark, minlength=D).double() / x
        V[table[row, j // page].long().cuda(), :, (j % page).cuda(), mark.cuda()] = one
    cache = rbs.PagedCache(K, V, torch.full((2 * hkv,), 448.0, device="cuda") if fp8 else None)
    Q = torch.randn(n, hq, D, generator=_gen(k)).to(torch.bfloat16).cuda().transpose(0, 1)
    lse = torch.full((hq, n), math.nan, device="cuda")
    O = rbs.rbs_paged_decode(rbs.make_shape(n, hq, hkv, 64), Q, cache, table.cuda(), _ints(lens), lse=lse)
    for row, x in enumerate(lens):
        o = O[:, row].cpu().double()
        err = (o - want[row]).abs()
        assert bool((err <= want[row] * (R.HALF_BF16 + 4 * R.U32)).all()), f"row {row}: a tile's mark"
        exact = math.log(x)
        step = 2.0 ** -23 * 2.0 ** math.floor(math.log2(max(math.log2(x), 1e-30)))
        tol = 2 * step * math.log(2) + 2 * R.U32 * exact
        assert tol < 0.75 * (math.log(x + 1) - exact)
        off = (lse[:, row].cpu().double() - exact).abs()
        assert bool((off <= tol).all()), f"row {row}: {float(off.max()):.3g} of {tol:.3g}"
