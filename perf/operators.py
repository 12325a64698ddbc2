"""The calls of a serving step over a paged key-value cache, in plain torch and through this package.

Four kinds of case, each one pass of a user's program for one attention layer:

  extend  pages for the new tokens of a batch of requests: block table, slots, positions
  rope    norm and rotation of a projection's queries and keys, keys and values put into the cache
  decode  attention of one new token per request over the cache
  step    the three one after another, as a decode step makes them

Head counts are those of the layers that the repository's workloads name (32 / 4 and 64 / 8, d = 128) and of
their tensor-parallel shards; lengths are those of chat turns, documents and 128K prompts.
"""

import math
import random

import torch

own = False

D = 128
EPS = 1e-6
E4M3_MAX = 448.0
#: Most cached tokens times KV heads (rows padded to the longest) and most projected values of a drawn case: the largest listed ones'.
MOST_CACHED = 32 * 16384 * 8
MOST_PROJECTED = 131072 * 40


def listed():
    return [
        # The bookkeeping of one decode step of a chat server's batch: a page every sixteenth token.
        dict(name="extend-decode-48", kind="extend", n=48, page=16, hi=8192, new=1),
        # The prompts of many requests admitted at once: pages and slots of some 64K tokens.
        dict(name="extend-prompts-200", kind="extend", n=200, page=64, hi=4096, new=650),
        # One user's next token: a single row, all latency.
        dict(name="rope-1-token", kind="rope", t=1, hq=32, hkv=4, page=16, fp8=False, rot=128, pairs="half", keep=False),
        # A decode batch of the 64-head layer with an FP8 cache.
        dict(name="rope-96-fp8", kind="rope", t=96, hq=64, hkv=8, page=32, fp8=True, rot=128, pairs="half", keep=False),
        # A prompt of odd length on a tensor-parallel shard; half of each head rotated, neighbours paired.
        dict(name="rope-3001-part", kind="rope", t=3001, hq=28, hkv=4, page=16, fp8=False, rot=64, pairs="next", keep=True),
        # The headline prompt, 128K tokens: the projection's output made ready for the sparse prefill and cached.
        dict(name="rope-128k", kind="rope", t=131072, hq=32, hkv=4, page=64, fp8=False, rot=128, pairs="half", keep=True),
        # A short chat's next token.
        dict(name="decode-1x700", kind="decode", n=1, lo=700, hi=700, hq=32, hkv=4, page=16, fp8=False, lse=False),
        # The first token after the headline prompt: one row, four KV heads, 128K keys.
        dict(name="decode-1x128k", kind="decode", n=1, lo=131071, hi=131071, hq=32, hkv=4, page=64, fp8=False, lse=False),
        # Ragged chats on a shard with groups of seven, with the log-sum-exp that a merge with other keys needs.
        dict(name="decode-24-chats", kind="decode", n=24, lo=1, hi=9000, hq=28, hkv=4, page=16, fp8=False, lse=True),
        # A throughput batch with an FP8 cache.
        dict(name="decode-200-fp8", kind="decode", n=200, lo=300, hi=2000, hq=32, hkv=4, page=32, fp8=True, lse=False),
        # Long documents on the 64-head layer: the most that one step reads.
        dict(name="decode-32-long", kind="decode", n=32, lo=9000, hi=16384, hq=64, hkv=8, page=128, fp8=False, lse=True),
        # A whole decode step of a batch.
        dict(name="step-64", kind="step", n=64, lo=500, hi=6000, hq=32, hkv=4, page=16, fp8=False, lse=False, rot=128, pairs="half"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["extend", "rope", "rope", "decode", "decode", "decode", "step"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "extend":
        new = rng.choice([1, 1, 0])
        n = _log_int(rng, 1, 512)
        return dict(kind=kind, n=n, page=page, hi=_log_int(rng, 100, 16384), new=new or _log_int(rng, 2, 262144 // (2 * n)))
    hq, hkv = rng.choice([(2, 1), (8, 1), (8, 8), (16, 2), (28, 4), (32, 4), (32, 4), (64, 8)])
    fp8 = rng.random() < 0.35
    rot, pairs = rng.choice([128, 128, 128, 64, 32]), rng.choice(["half", "half", "next"])
    if kind == "rope":
        t = _log_int(rng, 1, min(131072, MOST_PROJECTED // (hq + 2 * hkv)))
        return dict(kind=kind, t=t, hq=hq, hkv=hkv, page=page, fp8=fp8, rot=rot, pairs=pairs, keep=rng.random() < 0.5)
    hi = _log_int(rng, 30, 131072)
    n = _log_int(rng, 1, max(1, min(300, MOST_CACHED // (2 * hkv * hi))))
    case = dict(kind=kind, n=n, lo=max(1, int(hi * rng.choice([0.0, 0.2, 0.9]))), hi=hi, hq=hq, hkv=hkv, page=page, fp8=fp8,
                lse=rng.random() < 0.5)
    return case if kind == "decode" else dict(case, rot=rot, pairs=pairs)


# ------------------------------------------------------------------ inputs

def _spread(case, lo, hi, count):
    """The lengths of a case: spread over their logarithm, the longest among them, the same for every seed."""
    rng = random.Random(97 * count + 13 * hi + lo)
    out = [_log_int(rng, max(1, lo), hi) for _ in range(count)]
    out[count // 2] = hi
    return out


def _lengths(case):
    """Cached tokens of each row before the pass."""
    if case["kind"] == "extend":
        if case["new"] > 1:  # half the rows are new requests, the others are extended
            return [0 if s % 2 else x for s, x in enumerate(_spread(case, 10, case["hi"], case["n"]))]
        return _spread(case, 10, case["hi"], case["n"])
    return _spread(case, case["lo"], case["hi"], case["n"])


def _new(case):
    """New tokens of each row: one, or a prompt's of about new / 4 to new."""
    if case["kind"] == "extend" and case["new"] > 1:
        return _spread(case, max(1, case["new"] // 4), case["new"], case["n"])
    return [1] * case["n"]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _bookkeeping(case, gen):
    """Rows of a block table filled for the lengths, over a shuffled pool of pages, and the stack of free ones."""
    lens, new, p = _lengths(case), _new(case), case["page"]
    held = [-(-x // p) for x in lens]
    most = [-(-(x + a) // p) for x, a in zip(lens, new)]
    n, columns, pool = len(lens), max(most), sum(most) + 5
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(n, columns, dtype=torch.int32, device="cuda")
    cols = torch.arange(columns, device="cuda")
    held_t = torch.tensor(held, device="cuda")
    first = held_t.cumsum(0) - held_t
    inside = cols[None, :] < held_t[:, None]
    table[inside] = order[(first[:, None] + cols[None, :])[inside]]
    free = torch.zeros(pool, dtype=torch.int32, device="cuda")
    free[:pool - sum(held)] = order[sum(held):]
    return dict(table=table, free=free, n_free=_ints([pool - sum(held)]), lens=_ints(lens), new=_ints(new),
                pool=pool, most=sum(new) + (7 if sum(new) > n else 0), n=n)  # slots and positions of a padded batch


def _cache(case, pool, gen):
    """Keys around a mean per head and values around small offsets, in every place of every page."""
    hkv, p = case["hkv"], case["page"]
    z = torch.randn(hkv, 1, D, generator=gen, device="cuda")
    mu = 4.0 * z / z.norm(dim=-1, keepdim=True)
    kc = torch.empty(pool, hkv, p, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    kc.normal_(generator=gen)
    kc += mu.to(torch.bfloat16)
    vc.normal_(generator=gen)
    vc += 0.1 * torch.randn(hkv, 1, D, generator=gen, device="cuda").to(torch.bfloat16)
    amax = None
    if case["fp8"]:
        # The magnitude that maps to the largest E4M3 value; a few of the later tokens lie beyond it.
        amax = torch.cat([x[:1 + pool // 64].abs().amax(dim=(0, 2, 3)).float() for x in (kc, vc)])
        kc, vc = (_e4m3(x.float(), amax[i * hkv:(i + 1) * hkv, None, None]) for i, x in enumerate((kc, vc)))
    return kc, vc, amax


def _projection(t, hq, hkv, gen):
    """A projection's output [t][(hq + 2 hkv) d], seen as the (head, token, dimension) tensors that the package takes."""
    qkv = torch.empty(t, hq + 2 * hkv, D, dtype=torch.bfloat16, device="cuda")
    qkv.normal_(generator=gen)
    qkv *= torch.rand(1, hq + 2 * hkv, 1, generator=gen, device="cuda").add_(0.5).to(torch.bfloat16)
    x = qkv.transpose(0, 1)
    return x[:hq], x[hq:hq + hkv], x[hq + hkv:]


def _rotation(case, gen):
    """Norm weights, and frequencies of base 1e6 of which the slow ones are stretched fourfold (long contexts)."""
    rot = case["rot"]
    f = 1.0e6 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    turns = 32768 * f / (2 * math.pi)
    keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
    f = f * (keep + (1 - keep) / 4)
    weights = [(1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(torch.bfloat16) for _ in range(2)]
    return dict(f=f.float(), qw=weights[0], kw=weights[1], factor=0.1 * math.log(4.0) + 1, rot=rot, next=case["pairs"] == "next")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, s = case["kind"], dict(case=case)
    if kind in ("extend", "step"):
        s.update(_bookkeeping(case, gen))
    if kind == "rope":
        t, p = case["t"], case["page"]
        pool = -(-t // p) + 3
        order = torch.randperm(pool, generator=gen, device="cuda")
        start = (77 * t + 5) % 4096  # the rows of a prompt's later part, or of one request each
        far = torch.randint(0, 131072, (t,), generator=gen, device="cuda")
        s["positions"] = (start + torch.arange(t, device="cuda") if t > 512 else far).to(torch.int32)
        i = torch.arange(t, device="cuda")
        s["slots"] = (order[i // p] * p + i % p).to(torch.int32)
        s["pool"] = pool
    if kind == "decode":
        lens, p = _lengths(case), case["page"]
        held = torch.tensor([-(-x // p) for x in lens], device="cuda")
        s["pool"] = int(held.sum()) + 3
        order = torch.randperm(s["pool"], generator=gen, device="cuda").to(torch.int32)
        cols = torch.arange(int(held.max()), device="cuda")
        at = (held.cumsum(0) - held)[:, None] + cols[None, :]
        s["table"] = torch.where(cols[None, :] < held[:, None], order[at.clamp(max=s["pool"] - 1)], 0).to(torch.int32)
        s["lens"] = _ints(lens)
        s["n"] = len(lens)
        # Query rows of a token-major projection; logits with a standard deviation of about two.
        q = torch.randn(s["n"], case["hq"], D, generator=gen, device="cuda") * 2
        s["q"] = q.to(torch.bfloat16).transpose(0, 1)
    if kind in ("rope", "decode", "step"):
        s["kc"], s["vc"], s["amax"] = _cache(case, s["pool"], gen)
    if kind in ("rope", "step"):
        s["q_in"], s["k_in"], s["v_in"] = _projection(case["t"] if kind == "rope" else s["n"], case["hq"], case["hkv"], gen)
        s.update(_rotation(case, gen))
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"extend": _own_extend, "rope": _own_rope, "decode": _own_decode, "step": _own_step}[kind](state)
    return {"extend": _plain_extend, "rope": _plain_rope, "decode": _plain_decode, "step": _plain_step}[kind](state)


def _handles(s):
    """What a user's program makes once: the package's views of its buffers."""
    import paper_2609_20971_amd as rbs
    case = s["case"]
    if "free" in s:
        s["pages"] = rbs.Pages(s["table"], s["free"], s["n_free"], s["lens"], case["page"])
        s["out"] = rbs.PageStep.allocate(s["pages"], s["most"], in_place=False)
    if "kc" in s:
        s["cache"] = rbs.PagedCache(s["kc"], s["vc"], s["amax"])
        rows = s["q"].shape[1] if "q" in s else s["q_in"].shape[1]
        s["shape"] = rbs.make_shape(rows, case["hq"], case["hkv"], 128)
    if "f" in s:
        s["rope"] = rbs.Rope(s["f"], s["qw"], s["kw"], eps=EPS, interleaved=s["next"], factor=s["factor"])


def _own_extend(s):
    import paper_2609_20971_amd as rbs
    o = rbs.rbs_pages_extend(s["pages"], s["new"] if s["case"]["new"] > 1 else None, step=s["out"])
    return {"table": s["table"], "lens": o.seq_lens, "n_free": o.n_free, "cu": o.cu_tokens, "positions": o.positions,
            "slots": o.slots, "status": o.status}


def _own_rope(s):
    import paper_2609_20971_amd as rbs
    q, k = rbs.rbs_qk_norm_rope(s["shape"], s["rope"], s["q_in"], s["k_in"], s["positions"], V=s["v_in"], cache=s["cache"],
                                slots=s["slots"], keep_k=s["case"]["keep"])
    return _with_cache({"q": q, "k": k}, s)


def _own_decode(s):
    import paper_2609_20971_amd as rbs
    lse = torch.empty(s["case"]["hq"], s["n"], dtype=torch.float32, device="cuda") if s["case"]["lse"] else None
    return {"o": rbs.rbs_paged_decode(s["shape"], s["q"], s["cache"], s["table"], s["lens"], lse=lse), "lse": lse}


def _own_step(s):
    import paper_2609_20971_amd as rbs
    o = rbs.rbs_pages_extend(s["pages"], step=s["out"])
    q, _ = rbs.rbs_qk_norm_rope(s["shape"], s["rope"], s["q_in"], s["k_in"], o.positions, V=s["v_in"], cache=s["cache"],
                                slots=o.slots, keep_k=False)
    lse = torch.empty(s["case"]["hq"], s["n"], dtype=torch.float32, device="cuda") if s["case"]["lse"] else None
    out = rbs.rbs_paged_decode(s["shape"], q, s["cache"], s["table"], o.seq_lens, lse=lse)
    return _with_cache({"o": out, "lse": lse, "slots": o.slots, "lens": o.seq_lens}, s)


def _with_cache(out, s):
    f8 = torch.float8_e4m3fn
    out["kc"], out["vc"] = (x.view(f8) if s["case"]["fp8"] else x for x in (s["kc"], s["vc"]))
    return out


def _plain_extend(s):
    p, table, free = s["case"]["page"], s["table"], s["free"].long()
    lens, n_free = s["lens"].long(), s["n_free"].long()
    add = s["new"].long() if s["case"]["kind"] == "extend" and s["case"]["new"] > 1 else torch.ones_like(lens)
    add = torch.where(lens >= 0, add.clamp(min=0), 0)
    held, pages = (lens.clamp(min=0) + p - 1) // p, (lens.clamp(min=0) + add + p - 1) // p
    need = pages - held
    base = need.cumsum(0) - need
    cu = torch.nn.functional.pad(add.cumsum(0), (1, 0))
    status = (need.sum() > n_free).int() + 2 * (pages.max() > table.shape[1]).int() + 4 * (cu[-1] > s["most"]).int()
    ok = status == 0
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    fresh = (j >= held[:, None]) & (j < pages[:, None]) & ok
    source = n_free - 1 - base[:, None] - (j - held[:, None])
    table.copy_(torch.where(fresh, free[source.clamp(0, free.numel() - 1)].int(), table))
    t = torch.arange(s["most"], device="cuda")
    row = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=s["n"] - 1)
    inside = (t < cu[-1]) & ok
    at = torch.where(inside, lens[row] + t - cu[row], 0)
    slot = table[row, at // p].long() * p + at % p
    return {"table": table, "lens": torch.where(ok, lens + add, lens).int(), "n_free": (n_free - need.sum() * ok).int(),
            "cu": (cu * ok).int(), "positions": torch.where(inside, at, -1).int(),
            "slots": torch.where(inside, slot, -1).int(), "status": status.int()}


def _e4m3(x, amax):
    scale = torch.where(amax > 0, E4M3_MAX / amax, torch.ones_like(amax))
    return (x * scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes, amax):
    return codes.view(torch.float8_e4m3fn).float() * torch.where(amax > 0, amax / E4M3_MAX, torch.ones_like(amax))


def _plain_norm(x, w):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _plain_turn(x, cos, sin, rot, neighbours):
    if neighbours:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(-2) if neighbours else torch.cat([a, b], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_rotate(s, positions, slots):
    """Queries and keys ready, keys and values in the cache; returns q and k in bf16."""
    p, hkv = s["case"]["page"], s["case"]["hkv"]
    angle = positions.double()[:, None] * s["f"].double()
    cos, sin = angle.cos().float() * s["factor"], angle.sin().float() * s["factor"]
    q = _plain_turn(_plain_norm(s["q_in"], s["qw"]), cos, sin, s["rot"], s["next"]).to(torch.bfloat16)
    k = _plain_turn(_plain_norm(s["k_in"], s["kw"]), cos, sin, s["rot"], s["next"])
    page, place = slots.long() // p, slots.long() % p
    if s["amax"] is None:
        kept, v = k.to(torch.bfloat16), s["v_in"]
    else:
        kept, v = _e4m3(k, s["amax"][:hkv, None, None]), _e4m3(s["v_in"].float(), s["amax"][hkv:, None, None])
    s["kc"][page, :, place] = kept.transpose(0, 1)
    s["vc"][page, :, place] = v.transpose(0, 1)
    return q, k.to(torch.bfloat16)


def _plain_rope(s):
    q, k = _plain_rotate(s, s["positions"], s["slots"])
    return _with_cache({"q": q, "k": k if s["case"]["keep"] else None}, s)


def _plain_attend(s, q, lens):
    """One query row per request over its pages, gathered into rows of equal length and masked."""
    case, n = s["case"], s["n"]
    hq, hkv = case["hq"], case["hkv"]

    def gathered(x, amax):
        x = x[s["table"].long()].transpose(1, 2).reshape(n, hkv, -1, D)
        return x.float() if amax is None else _values(x, amax[:, None, None])

    a = s["amax"]
    k = gathered(s["kc"], None if a is None else a[:hkv])
    rows = q.transpose(0, 1).reshape(n, hkv, hq // hkv, D).float()
    logits = torch.matmul(rows, k.transpose(-1, -2)) / math.sqrt(D)
    outside = torch.arange(k.shape[2], device="cuda")[None, :] >= lens[:, None]
    logits = logits.masked_fill(outside[:, None, None, :], -math.inf)
    del k
    top = logits.amax(-1, keepdim=True)
    e = torch.exp(logits - top)
    del logits
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, gathered(s["vc"], None if a is None else a[hkv:])) / total
    out = out.reshape(n, hq, D).transpose(0, 1).to(torch.bfloat16)
    lse = (top + total.log()).reshape(n, hq).transpose(0, 1).contiguous()
    return {"o": out, "lse": lse if case["lse"] else None}


def _plain_decode(s):
    return _plain_attend(s, s["q"], s["lens"])


def _plain_step(s):
    pages = _plain_extend(s)
    q, _ = _plain_rotate(s, pages["positions"], pages["slots"])
    out = _plain_attend(s, q, pages["lens"])
    return _with_cache(dict(out, slots=pages["slots"], lens=pages["lens"]), s)


# ------------------------------------------------------------------ what a pass cannot do without

def _extend_bytes(case):
    lens, new, p = _lengths(case), _new(case), case["page"]
    fresh = sum(-(-(x + a) // p) - -(-x // p) for x, a in zip(lens, new))
    touched = sum(-(-(x + a) // p) - x // p for x, a in zip(lens, new))
    # Lengths in and out, counts, offsets; a free page read and its entry written; entries read; position and slot.
    return 4 * (4 * case["n"] + 8) + 8 * fresh + 4 * (touched - fresh) + 8 * sum(new)


def _rope_bytes(case, t, keep):
    width = 1 if case["fp8"] else 2
    moved = t * D * (2 * (2 * case["hq"] + 2 * case["hkv"]) + 2 * case["hkv"] * width + (2 * case["hkv"] if keep else 0))
    return moved + 8 * t + 4 * D + 2 * case["rot"] + (8 * case["hkv"] if case["fp8"] else 0)


def work(case):
    kind = case["kind"]
    if kind == "extend":
        return {"bytes": _extend_bytes(case), "flops": 0}
    if kind == "rope":
        return {"bytes": _rope_bytes(case, case["t"], case["keep"]), "flops": 10 * case["t"] * D * (case["hq"] + case["hkv"])}
    lens = [x + (kind == "step") for x in _lengths(case)]
    n, hq, hkv, p = case["n"], case["hq"], case["hkv"], case["page"]
    moved = sum(lens) * hkv * D * 2 * (1 if case["fp8"] else 2) + 4 * n * hq * D + 4 * n
    moved += 4 * sum(-(-x // p) for x in lens) + (4 * hq * n if case["lse"] else 0)
    flops = 4 * hq * D * sum(lens)
    if kind == "step":
        moved += _extend_bytes(case) + _rope_bytes(case, n, False)
        flops += 10 * n * D * (hq + hkv)
    return {"bytes": moved, "flops": flops}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "extend":
        r = _exact_extend(s)
        return {x: torch.tensor(r[x], dtype=torch.int32) for x in
                ("table", "lens", "n_free", "cu", "positions", "slots", "status")}
    if kind == "rope":
        q, k, kc, vc = _exact_rotate(s, s["positions"].tolist(), s["slots"])
        return {"q": q, "k": k if case["keep"] else None, "kc": kc, "vc": vc}
    if kind == "decode":
        kc, vc = _exact_cache(s)
        return _exact_attend(s, s["q"].double(), kc, vc, s["table"].tolist(), s["lens"].tolist())
    r = _exact_extend(s)
    q, _, kc, vc = _exact_rotate(s, r["positions"], torch.tensor(r["slots"], device="cuda"))
    # The step's attention reads the rotated queries and the cache as they are held, rounded to their types.
    q = q.to(torch.bfloat16).double()
    if case["fp8"]:
        held = [x.float().to(torch.float8_e4m3fn).double() * f for x, f in zip((kc, vc), _exact_factors(s))]
    else:
        held = [x.to(torch.bfloat16).double() for x in (kc, vc)]
    out = _exact_attend(s, q, *held, r["table"], r["lens"])
    return {"o": out["o"], "lse": out["lse"], "slots": torch.tensor(r["slots"], dtype=torch.int32),
            "lens": torch.tensor(r["lens"], dtype=torch.int32), "kc": kc, "vc": vc}


def _exact_extend(s):
    """The bookkeeping of one request after another, with a list for the stack."""
    p = s["case"]["page"]
    table, lens, counts = s["table"].tolist(), s["lens"].tolist(), s["new"].tolist()
    stack = s["free"].tolist()[:int(s["n_free"])]
    cu, positions, slots = [0], [], []
    for row, count in enumerate(counts):
        for _ in range(count):
            at = lens[row]
            if at % p == 0:
                table[row][at // p] = stack.pop()
            positions.append(at)
            slots.append(table[row][at // p] * p + at % p)
            lens[row] += 1
        cu.append(len(positions))
    behind = [-1] * (s["most"] - len(slots))
    return dict(table=table, lens=lens, n_free=[len(stack)], cu=cu, positions=positions + behind, slots=slots + behind, status=[0])


def _exact_factors(s):
    """What a code of each head's keys and values is multiplied by, as [hkv, 1, 1] tensors."""
    hkv = s["case"]["hkv"]
    return [(s["amax"][i * hkv:(i + 1) * hkv].double() / E4M3_MAX)[:, None, None] for i in range(2)]


def _exact_cache(s):
    if s["amax"] is None:
        return s["kc"], s["vc"]
    return [x.view(torch.float8_e4m3fn).to(torch.bfloat16).double() * f for x, f in zip((s["kc"], s["vc"]), _exact_factors(s))]


def _exact_rotate(s, positions, slots):
    """As complex numbers: a pair is a number, a rotation the product with one of length `factor`."""
    case = s["case"]
    p, rot, hkv = case["page"], s["rot"], case["hkv"]
    at = torch.tensor(positions, dtype=torch.float64, device="cuda")
    spin = torch.polar(torch.full((), s["factor"], dtype=torch.float64, device="cuda").expand(at.numel(), rot // 2),
                       at[:, None] * s["f"].double()[None, :])

    def ready(x, w):
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for h in range(x.shape[0]):
            y = x[h].double()
            y = y / (y.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
            if s["next"]:
                first, second = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
            else:
                first, second = torch.arange(rot // 2), torch.arange(rot // 2, rot)
            z = torch.complex(y[:, first].contiguous(), y[:, second].contiguous()) * spin
            y[:, first], y[:, second] = z.real, z.imag
            out[h] = y
        return out

    q, k, v = ready(s["q_in"], s["qw"]), ready(s["k_in"], s["kw"]), s["v_in"].double()
    if s["amax"] is None:
        kc, vc = s["kc"].double(), s["vc"].double()
    else:  # in units of the codes, as the cache is returned
        kc, vc = (x.view(torch.float8_e4m3fn).to(torch.bfloat16).double() for x in (s["kc"], s["vc"]))
        kf, vf = _exact_factors(s)
        k_kept, v_kept = (k / kf).clamp(-E4M3_MAX, E4M3_MAX), (v / vf).clamp(-E4M3_MAX, E4M3_MAX)
    flat = slots.long().to("cuda")
    for h in range(hkv):
        kc[:, h][flat // p, flat % p] = k[h] if s["amax"] is None else k_kept[h]
        vc[:, h][flat // p, flat % p] = v[h] if s["amax"] is None else v_kept[h]
    return q, k, kc, vc


def _exact_attend(s, q, kc, vc, table, lens):
    case, p = s["case"], s["case"]["page"]
    hq, hkv = case["hq"], case["hkv"]
    group = hq // hkv
    out = torch.zeros(hq, len(lens), D, dtype=torch.float64, device="cuda")
    lse = torch.full((hq, len(lens)), -math.inf, dtype=torch.float64, device="cuda")
    for row, length in enumerate(lens):
        pages = torch.tensor(table[row][:-(-length // p)], device="cuda", dtype=torch.long)
        k, v = kc[pages], vc[pages]
        for g in range(hkv):
            keys, values = (x[:, g].reshape(-1, D)[:length].double() for x in (k, v))
            heads = slice(g * group, (g + 1) * group)
            logits = q[heads, row] @ keys.T / math.sqrt(D)
            lse[heads, row] = torch.logsumexp(logits, -1)
            out[heads, row] = torch.softmax(logits, -1) @ values
    return {"o": out, "lse": lse if case["lse"] else None}
