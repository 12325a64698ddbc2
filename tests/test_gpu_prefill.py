"""GPU: attention of all new tokens of a batch over a paged cache against a plain
implementation in 64 bits (tests/cache_reference.py)."""

from __future__ import annotations

import math

import pytest
import torch

import paper_2609_20971_amd as rbs
from tests import cache_reference as C
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

D = 128


def _say(*a):
    print(*a, flush=True)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _case(rows, hq, hkv, page, fmt, layout, seed, spare=0, bad="nan", k_scale=1.0, columns=1):
    """rows: (cached tokens before, new tokens), or None for an unused row, or (length, None) for one without new tokens."""
    g = _gen(seed)
    lens = [-1 if r is None else r[0] + (r[1] or 0) for r in rows]
    new = [0 if r is None else r[1] or 0 for r in rows]
    n = len(rows)
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
    V = torch.randn(pool, hkv, page, D, generator=g) + 0.2
    amax = torch.rand(2 * hkv, generator=g) * 3 + 2
    cache = C.cache_of(K, V, live, fmt, layout, amax, bad)
    cu = [0]
    for a in new:
        cu.append(cu[-1] + a)
    t = max(1, cu[-1] + spare)
    q = (torch.randn(t, hq, D, generator=g) * 1.5).to(torch.bfloat16)
    return dict(cache=cache, table=table, lens=lens, new=new, cu=cu, q=q, page=page, hq=hq, hkv=hkv, fmt=fmt, t=t)


def _run(c, scale=0.0, q_layout="tokens", lse=True, cu=None, **more):
    q = c["q"].cuda()
    if q_layout == "heads":
        Q = q.transpose(0, 1).contiguous()
    elif q_layout == "tokens":
        Q = q.transpose(0, 1)
    else:  # a fused projection's part
        Q = torch.cat([q, q[:, :1].expand(-1, 2 * c["hkv"], -1)], 1).transpose(0, 1)[:c["hq"]]
    O = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device="cuda").fill_(7.0)
    l = torch.full((c["hq"], c["t"]), 7.0, device="cuda") if lse else None
    got = rbs.rbs_paged_prefill(rbs.make_shape(c["t"], c["hq"], c["hkv"], 64), Q, c["cache"], c["table"].cuda(), _ints(c["lens"]),
                                _ints(c["cu"] if cu is None else cu), scale, O=O, lse=l, **more)
    assert got is O
    return O, l


def _check(c, O, lse, scale, rows=None):
    K, V = C.cache_values(c["cache"])
    written = torch.zeros(c["t"], dtype=torch.bool)
    worst = 0.0
    O, lse = O.cpu().double(), None if lse is None else lse.cpu().double()
    for row, (n, a) in enumerate(zip(c["lens"], c["new"])):
        if n < 0 or a == 0:
            continue
        at = slice(c["cu"][row], c["cu"][row + 1])
        written[at] = True
        if rows is not None and row not in rows:
            continue
        k, v = (R.gather(x, c["table"][row], n, c["page"]) for x in (K, V))
        last = n - a + torch.arange(a)
        o, l, o_tol, l_tol = C.attend(c["q"][at].double().transpose(0, 1), k, v, scale, last, one_part=True)
        err = (O[:, at] - o).abs()
        share = (err / o_tol.clamp(min=1e-38))
        assert bool((err <= o_tol).all()), f"row {row} ({n - a} + {a}): {share.max():.3f} of the tolerance at {divmod(int(share.argmax()) // D, a)}"
        worst = max(worst, float(share.max()))
        if lse is not None:
            empty = l == -math.inf
            assert bool((lse[:, at][empty] == -math.inf).all())
            assert bool(((lse[:, at] - l).abs() <= l_tol)[~empty].all()), f"row {row}: lse"
    assert bool((O[:, ~written] == 7.0).all()) and (lse is None or bool((lse[:, ~written] == 7.0).all())), "tokens of no row were written"
    return worst


ROWS = [
    # rows (before, new), heads, page, format, cache layout, q layout, tokens to spare, scale
    ([(0, 1)], 2, 1, 16, "bf16", "heads", "heads", 0, 0.0),
    ([(0, 5)], 1, 1, 16, "fp8", "tokens", "tokens", 3, 0.0),
    ([(0, 17)], 8, 1, 16, "fp4", "heads", "qkv", 0, 0.0),
    ([(0, 127), (0, 128), (0, 129), (0, 1)], 4, 4, 32, "bf16", "heads", "tokens", 0, 0.3),
    ([(3, 40), None, (200, None), (0, 1), (255, 2), (256, 16), (1000, 3)], 28, 4, 16, "bf16", "tokens", "tokens", 9, 0.0),
    ([(3, 40), None, (200, None), (0, 1), (255, 2), (256, 16), (1000, 3)], 28, 4, 16, "fp8", "tokens", "qkv", 9, 0.0),
    ([(3, 40), None, (200, None), (0, 1), (255, 2), (256, 16), (1000, 3)], 28, 4, 16, "fp4", "tokens", "heads", 9, 0.0),
    ([(127, 1), (128, 1), (126, 3), (0, 300)], 16, 2, 64, "bf16", "heads", "tokens", 0, 0.0),
    ([(0, 700)], 6, 3, 128, "fp8", "heads", "heads", 0, 0.0),
    ([(77, 500), (500, 77)], 7, 1, 256, "fp4", "heads", "tokens", 1, 0.0),
    ([(4000, 4), (3000, 5), (10, 6), (0, 3), (6000, 1)], 8, 2, 16, "bf16", "heads", "tokens", 0, 0.0),       # split
    ([(4000, 4), (3000, 5), (10, 6), (0, 3), (6000, 1)], 8, 2, 32, "fp8", "tokens", "tokens", 0, 0.0),
    ([(4000, 4), (3000, 5), (10, 6), (0, 3), (6000, 1)], 8, 2, 64, "fp4", "heads", "tokens", 2, 0.0),
    ([(20000, 1)], 8, 1, 64, "bf16", "heads", "tokens", 0, 0.0),
    ([(9000, 33)], 32, 4, 64, "bf16", "heads", "tokens", 0, 0.0),
    ([(50, 2)] * 300 + [None] * 30 + [(0, 1)] * 20, 8, 2, 16, "bf16", "heads", "tokens", 5, 0.0),              # two rows a thread
    ([(i % 37, 1 + i % 3) for i in range(1500)] + [(9, None)] * 2000, 4, 2, 16, "fp4", "heads", "tokens", 0, 0.0),
    ([(0, 300)], 512, 512, 16, "bf16", "heads", "tokens", 0, 0.0),                                              # more tiles than room
    ([(0, 3)], 512, 1, 16, "bf16", "tokens", "tokens", 0, 0.0),                                                 # a token's heads over four tiles
    ([(900, 40)], 130, 2, 16, "fp8", "heads", "tokens", 0, 0.0),
    ([(0, 1500), (0, 37), (700, 900)], 32, 8, 16, "bf16", "heads", "qkv", 0, 0.0),
    ([(0, 2600)], 32, 4, 128, "fp4", "heads", "tokens", 0, 0.0),                                                # whole tiles
    ([(0, 2600)], 32, 4, 16, "fp8", "heads", "tokens", 0, 0.0),
    ([(0, 2600), (31, 2)], 32, 4, 16, "bf16", "heads", "tokens", 0, 0.0),
    # At most 32 queries to a row, whole rows to a unit (the longest past 4096 keys).
    ([(9000, 3), (31, 1), (32, 1), (28, 4), (0, 32), (5, 27)] + [(20, 2)] * 66, 8, 8, 16, "bf16", "heads", "tokens", 0, 0.0),
    ([(9000, 3), (31, 1), (32, 1), (28, 4), (0, 32), (5, 27)] + [(20, 2)] * 66, 8, 8, 32, "fp8", "heads", "heads", 3, 0.0),
    ([(9000, 3), (31, 1), (32, 1), (28, 4), (0, 32), (5, 27)] + [(20, 2)] * 66, 8, 8, 16, "fp4", "tokens", "qkv", 0, 0.0),
    ([(2500, 32), (2500, 33), (95, 32), (96, 1)], 4, 4, 16, "fp4", "heads", "tokens", 0, 0.0),
    ([(2500, 4), (2500, 5), (90, 2)], 28, 4, 16, "bf16", "heads", "tokens", 0, 0.0),
    # Split, among more rows than a wave has lanes.
    ([(9, None)] * 70 + [(6000, 3), None, (0, 200), (3000, 40)] + [None] * 30, 8, 2, 16, "bf16", "heads", "tokens", 4, 0.0),
    ([(9, None)] * 70 + [(6000, 3), None, (0, 200), (3000, 40)] + [None] * 30, 8, 2, 32, "fp8", "tokens", "tokens", 0, 0.0),
    ([(6000, 3), None, (0, 200), (3000, 40)] + [None] * 4000 + [(500, 1)], 8, 2, 16, "fp4", "heads", "heads", 0, 0.0),
]


@pytest.mark.parametrize("k", range(len(ROWS)))
def test_prefill(k):
    rows, hq, hkv, page, fmt, layout, q_layout, spare, scale = ROWS[k]
    _say(f"[prefill] {len(rows)} rows, heads {hq}/{hkv}, page {page}, {fmt}")
    c = _case(rows, hq, hkv, page, fmt, layout, 300 + k, spare)
    O, lse = _run(c, scale, q_layout)
    busy = [i for i, r in enumerate(rows) if r is not None and r[1] is not None]
    some = None if len(busy) < 40 else set(busy[:6]) | set(busy[::17])
    _say(f"[prefill] {_check(c, O, lse, scale if scale > 0 else 1 / math.sqrt(D), some):.3f} of the tolerance")
    O2, _ = _run(c, scale, q_layout, lse=False)
    assert torch.equal(O, O2), "the same call again"


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("rows", [[(100, 60), (0, 33)], [(5000, 3)], [(0, 2700)]])
def test_later_tokens_do_not_reach_earlier_ones(rows, fmt):
    """Values and keys that are not finite at later positions leave earlier tokens' results as they were, bit for bit."""
    c = _case(rows, 32, 4, 16, fmt, "heads", 41)
    clean, clean_lse = _run(c)
    before, new = rows[0]
    cache, page = c["cache"], 16
    for i in sorted({1, new // 2, new - 1}):  # this token's value, and the next one's key
        for buf, at, head in ((("V", "V_scale")[fmt == "fp4"], before + i, 1), (("K", "K_scale")[fmt == "fp4"], before + i, 2)):
            p, place = int(c["table"][0, at // page]), at % page
            t = getattr(cache, buf)
            if fmt == "bf16":
                t[p, head, place, 5] = math.nan if i % 2 else math.inf
                t[p, head, place, 77] = -math.inf
            elif fmt == "fp8":
                t[p, head, place, 5] = 0x7F
            else:
                t[p, head, place, 2] = 255
    O, lse = _run(c)
    touched = sorted({1, new // 2, new - 1})
    first = touched[0]
    assert torch.equal(O[:, :first], clean[:, :first]) and torch.equal(lse[:, :first], clean_lse[:, :first])
    assert torch.equal(O[:8], clean[:8]) and torch.equal(O[24:], clean[24:])          # other heads
    assert torch.equal(O[:, new:], clean[:, new:])                                     # other rows
    for i in range(first, new):
        assert bool((~O[8:16, i].isfinite()).any()), i       # an attended value reaches its elements
        assert bool(O[16:24, i].isnan().all()), i            # an attended key the whole result
    element = 70 if fmt != "fp4" else 3
    assert torch.equal(O[8:16, :, element], clean[8:16, :, element])


def test_infinite_values_are_attended():
    """An infinite value that a token attends makes that element infinite, of the masked block too."""
    c = _case([(0, 100)], 8, 1, 16, "bf16", "heads", 42)
    c["cache"].V[int(c["table"][0, 2]), 0, 3, 9] = math.inf    # position 35
    c["cache"].V[int(c["table"][0, 3]), 0, 0, 9] = -math.inf   # position 48: NaN from here on
    O, _ = _run(c)
    assert bool(O[:, :35].isfinite().all())
    assert bool((O[:, 35:48, 9] == math.inf).all()) and bool(O[:, 48:, 9].isnan().all())
    O[:, :, 9] = 0
    assert bool(O.isfinite().all())


def test_infinite_values_of_few_queries():
    """The same where the waves divide the keys: 4 heads of 8 tokens; position 35 is attended by the last three."""
    c = _case([(30, 8)], 4, 1, 16, "bf16", "heads", 49)
    c["cache"].V[int(c["table"][0, 2]), 0, 3, 9] = math.inf    # position 35
    c["cache"].V[int(c["table"][0, 0]), 0, 7, 70] = -math.inf  # position 7: attended by all
    O, lse = _run(c)
    assert bool(O[:, :5, 9].isfinite().all()) and bool((O[:, 5:, 9] == math.inf).all())
    assert bool((O[:, :, 70] == -math.inf).all()) and bool(lse.isfinite().all())
    O[:, :, 9] = O[:, :, 70] = 0
    assert bool(O.isfinite().all())


def test_large_logits():
    c = _case([(700, 50), (0, 33), (4000, 9)], 8, 2, 16, "bf16", "heads", 43, k_scale=12.0, bad="large")
    O, lse = _run(c, 2.0)
    _check(c, O, lse, 2.0)


def test_one_token_rows_are_decode_rows():
    """A single new token a row gives what the decode call gives, up to the rounding of the weights."""
    lens = [1, 17, 300, 1025, 4000]
    c = _case([(n - 1, 1) for n in lens], 16, 2, 16, "bf16", "heads", 44)
    O, lse = _run(c)
    Q = c["q"].cuda().transpose(0, 1)
    l2 = torch.empty_like(lse)
    O2 = rbs.rbs_paged_decode(rbs.make_shape(5, 16, 2, 64), Q, c["cache"], c["table"].cuda(), _ints(lens), lse=l2)
    assert bool(((O.float() - O2.float()).abs() <= 2 ** -7 * 4).all())
    assert torch.allclose(lse, l2, atol=2.0 ** -8)
    _check(c, O, lse, 1 / math.sqrt(D))


def test_more_new_tokens_than_cached_ones():
    """Tokens before their row's first key: zeros, and -inf."""
    c = _case([(0, 40), (3, 7)], 4, 2, 16, "bf16", "heads", 45)
    full, full_lse = _run(c)
    c["lens"] = [25, 0]
    O, lse = _run(c)
    assert bool((O[:, :15] == 0).all()) and bool((lse[:, :15] == -math.inf).all())
    assert bool((O[:, 40:] == 0).all()) and bool((lse[:, 40:] == -math.inf).all())
    k = C.cache_values(c["cache"])
    o, l, o_tol, l_tol = C.attend(c["q"][15:40].double().transpose(0, 1), *(R.gather(x, c["table"][0], 25, 16) for x in k),
                                  1 / math.sqrt(D), torch.arange(25), one_part=True)
    assert bool(((O[:, 15:40].cpu().double() - o).abs() <= o_tol).all())
    assert bool(((lse[:, 15:40].cpu().double() - l).abs() <= l_tol).all())


def test_clamps_lengths_and_pages():
    """Lengths past the table and page numbers outside the cache stay inside the buffers."""
    c = _case([(60, 4), (0, 64)], 4, 2, 16, "bf16", "heads", 46, columns=0)
    want, _ = _run(c)
    pool = c["cache"].K.shape[0]
    wild, tame = (dict(c, table=c["table"].clone()) for _ in range(2))
    wild["table"][0, 1], wild["table"][0, 2] = 2**31 - 1, -2**31
    tame["table"][0, 1], tame["table"][0, 2] = pool - 1, 0
    assert torch.equal(_run(wild)[0].nan_to_num(3.0), _run(tame)[0].nan_to_num(3.0))
    long = dict(c, lens=[2**31 - 1, 64])  # all its tokens lie past the table: they attend all of it
    got, _ = _run(long)
    assert torch.equal(got[:, 4:], want[:, 4:])
    o = [C.attend(c["q"][:4].double().transpose(0, 1), *(R.gather(x, c["table"][0], 64, 16) for x in C.cache_values(c["cache"])),
                  1 / math.sqrt(D), torch.full((4,), 63), one_part=True)][0]
    assert bool(((got[:, :4].cpu().double() - o[0]).abs() <= o[2]).all())


def test_offsets_that_are_none():
    """Offsets outside Q leave their row out; where they descend, no row has any tokens."""
    c = _case([(10, 6), (20, 7), (5, 8)], 4, 2, 16, "bf16", "heads", 47)
    want, _ = _run(c)
    out, lse = _run(c, cu=[0, 6, 13, 22])  # the last row's end is past Q
    assert torch.equal(out[:, :13], want[:, :13]) and bool((out[:, 13:] == 7.0).all()) and bool((lse[:, 13:] == 7.0).all())
    out, _ = _run(c, cu=[-1, 6, 13, 21])
    assert torch.equal(out[:, 6:], want[:, 6:]) and bool((out[:, :6] == 7.0).all())
    for cu in ([0, 13, 6, 21], [21, 0, 21, 0], [5, 4, 3, 2], [2**31 - 1, -2**31, 0, 21]):
        out, lse = _run(c, cu=cu)
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all()), cu
    out, _ = _run(c, cu=[0, 0, 0, 0])
    assert bool((out == 7.0).all())


def test_pages_past_32_bits():
    page, hkv, hq = 256, 8, 16
    for fmt, k in (("bf16", 1), ("fp4", 4)):
        n_pages = k * (1 << 31) // (page * hkv * D) + 40
        c = _case([(5000, 30), (0, 300)], hq, hkv, page, fmt, "heads", 48)
        small = c["cache"].K.shape[0]
        far = rbs.PagedCache.allocate(n_pages, page, hkv, fp4=fmt == "fp4")
        assert far.K.numel() * far.K.element_size() >= 1 << 32
        for name in ("K", "V", "K_scale", "V_scale")[:4 if fmt == "fp4" else 2]:
            getattr(far, name)[-small:] = getattr(c["cache"], name)
        moved = dict(c, cache=far, table=torch.where(c["table"] >= 0, c["table"] + n_pages - small, c["table"]))
        want, got = _run(c), _run(moved)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del far, moved
        torch.cuda.empty_cache()


def test_longest_row():
    """A table of nearly 2^31 places, all of one page, and a length past it: every key 0 and every value 1, so that all
    weights are 1 and the sums whole numbers (exact in a piece, of at most 2^22 + 64 keys, and off by a rounding each
    where 512 pieces are joined)."""
    page, columns = 256, 2 ** 23 - 1
    cache = rbs.PagedCache.allocate(1, page, 1)
    cache.K.zero_()
    cache.V.fill_(1.0)
    table = torch.zeros(1, columns, dtype=torch.int32, device="cuda")
    Q = torch.randn(2, 8, D, generator=_gen(77)).to(torch.bfloat16).cuda().transpose(0, 1)
    lse = torch.empty(8, 2, device="cuda")
    O = rbs.rbs_paged_prefill(rbs.make_shape(2, 8, 1, 64), Q, cache, table, _ints([2 ** 31 - 1]), _ints([0, 2]), lse=lse)
    assert bool((O == 1.0).all())
    want = math.log(columns * page)
    # The sum: 516 roundings; log2 and the change of base: 2 steps of the result's 31 each.
    assert bool(((lse.cpu().double() - want).abs() <= 516 * R.U32 + 4 * want * R.U32).all())
