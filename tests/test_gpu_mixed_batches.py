"""GPU: the calls of a server together, as it would make them: room for new tokens, norm
and rotation into the cache, attention of prompts, parts of prompts, drafted and
single tokens in one batch, decode steps, and rows moved between caches; eager, captured,
from several threads and on streams given by name."""

from __future__ import annotations

import math
import threading

import pytest
import torch

import paper_2609_20971_amd as rbs
from paper_2609_20971_amd import _paged as P
from tests import cache_reference as C
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

D, HQ, HKV, PAGE, ROWS, ROOM = 128, 8, 2, 16, 6, 900
SCALE = 1 / math.sqrt(D)
FORMATS = ["bf16", "fp8", "fp4"]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _qkv(n, seed):
    """Parts of one projection's output."""
    x = torch.randn(n, HQ + 2 * HKV, D, generator=_gen(seed)).to(torch.bfloat16).cuda().transpose(0, 1)
    return x[:HQ], x[HQ:HQ + HKV], x[HQ + HKV:]


def _rope():
    w = (torch.rand(D, generator=_gen(5)) + 0.5).to(torch.bfloat16).cuda()
    return rbs.Rope(*rbs.rope_frequencies()[:1], w, w)


class Server:
    """Six rows; every step's tokens lie in buffers for ROOM tokens."""

    def __init__(self, fmt, rope, now):
        amax = torch.full((2 * HKV,), 7.0).cuda() if fmt == "fp8" else None
        self.fmt, self.rope, self.now = fmt, rope, now
        self.pages = rbs.Pages.allocate(ROWS, 400, 600, PAGE)
        self.cache = C.make_cache(600, HKV, PAGE, fmt, amax=amax, fill=0xFF)  # NaN everywhere
        self.out = rbs.PageStep.allocate(self.pages, ROOM)
        self.counts = _ints([0] * ROWS)
        self.shape = rbs.make_shape(ROOM, HQ, HKV, 64)
        self.O = torch.empty(ROOM, HQ, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        self.lse = torch.empty(HQ, ROOM, device="cuda")
        self.O1, self.lse1 = torch.empty_like(self.O), torch.empty_like(self.lse)
        self.read = torch.empty(2, HKV, ROOM, D, dtype=torch.bfloat16, device="cuda")
        self.pages.seq_lens.copy_(_ints([0, -1, 0, 0, -1, 0]))

    def step(self):
        """The batch's attention twice (all tokens; only the rows' last ones), and its tokens read back from the cache."""
        Q, K, V = self.now
        for x in (self.O, self.lse, self.O1, self.lse1, self.read):
            x.fill_(7.0)
        before = self.pages.seq_lens.clone()
        o = rbs.rbs_pages_extend(self.pages, self.counts, step=self.out)
        self.q, _ = rbs.rbs_qk_norm_rope(self.shape, self.rope, Q, K, o.positions, V=V, cache=self.cache, slots=o.slots, keep_k=False)
        table = self.pages.page_table
        rbs.rbs_paged_prefill(self.shape, self.q, self.cache, table, o.seq_lens, o.cu_tokens, O=self.O, lse=self.lse)
        rbs.rbs_paged_decode(self.shape, self.q, self.cache, table, o.seq_lens, O=self.O1, lse=self.lse1, cu_tokens=o.cu_tokens)
        rbs.rbs_cache_read(self.shape, self.cache, table, o.cu_tokens, before, *self.read)

    def outputs(self):
        return [x.clone() for x in (self.O, self.lse, self.O1, self.lse1, self.read)]


# New tokens of the rows: prompts; the next part of one and single tokens; drafts; a long part; none at all.  (Rows 1
# and 4 are admitted with the third step, row 3 is released before the last but one.)
STEPS = [[300, 9, 17, 0, 9, 1], [500, 0, 1, 380, 0, 1], [4, 1, 5, 3, 130, 0], [890, 1, 1, 1, 1, 1], [0] * 6, [1, 3, 1, 9, 4, 2]]


def _between(server, k):
    if k == 2:
        server.pages.seq_lens[1] = 0
        server.pages.seq_lens[4] = 0
    if k == 4:
        rbs.rbs_pages_release(server.pages, _ints([0, 0, 0, 1, 0, 0]))
    server.counts.copy_(_ints(STEPS[k]))


def _check(server, k):
    """Every row's tokens against the formula, over the cache's contents."""
    fmt, lens = server.fmt, server.pages.seq_lens.tolist()
    assert server.out.status.tolist() == [0]
    cu, table = server.out.cu_tokens.tolist(), server.pages.page_table.cpu()
    K, V = C.cache_values(server.cache)
    O, lse, O1, lse1 = (x.cpu().double() for x in (server.O, server.lse, server.O1, server.lse1))
    read, q = server.read.cpu(), server.q.cpu().double()
    last_ones = []
    for row in range(ROWS):
        n, a = lens[row], cu[row + 1] - cu[row]
        assert a == (STEPS[k][row] if n >= 0 else 0)
        if a == 0:
            continue
        at = slice(cu[row], cu[row + 1])
        keys, values = (R.gather(x, table[row], n, PAGE) for x in (K, V))
        o, l, o_tol, l_tol = C.attend(q[:, at], keys, values, SCALE, n - a + torch.arange(a), one_part=True)
        assert bool(((O[:, at] - o).abs() <= o_tol).all()), f"step {k}, row {row}"
        assert bool(((lse[:, at] - l).abs() <= l_tol).all()), f"step {k}, row {row}"
        t = cu[row + 1] - 1
        last_ones.append(t)
        o, l, o_tol, l_tol = C.attend(q[:, t:t + 1], keys, values, SCALE, torch.tensor([n - 1]))
        assert bool(((O1[:, t:t + 1] - o).abs() <= o_tol).all()) and bool(((lse1[:, t:t + 1] - l).abs() <= l_tol).all())
        for got, held in zip(read, (keys, values)):
            held = held[:, n - a:]
            # (FP8: one rounding of the product, and one of the factor in fp32.)
            tol = 0.0 if fmt != "fp8" else held.abs() * (2.0 ** -8 + 2.0 ** -22)
            assert bool(((got[:, at].double() - held).abs() <= tol).all())
    rest = torch.ones(ROOM, dtype=torch.bool)
    rest[:cu[-1]] = False
    assert bool((O[:, rest] == 7.0).all()) and bool((lse[:, rest] == 7.0).all()) and bool((read[:, :, rest] == 7.0).all())
    rest[:] = True
    rest[last_ones] = False
    assert bool((O1[:, rest] == 7.0).all()) and bool((lse1[:, rest] == 7.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_steps_of_mixed_batches(fmt):
    """Each step against the formula; then the same steps as replays of one captured graph, with eager calls between
    them, equal to the eager ones bit for bit."""
    rope, inputs = _rope(), [_qkv(ROOM, 60 + k) for k in range(len(STEPS))]
    now = tuple(x.clone() for x in inputs[0])
    eager, want = Server(fmt, rope, now), []
    for k in range(len(STEPS)):
        _between(eager, k)
        for x, y in zip(now, inputs[k]):
            x.copy_(y)
        eager.step()
        _check(eager, k)
        want.append(eager.outputs())
    captured = Server(fmt, rope, now)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        captured.step()
    for k in range(len(STEPS)):
        _between(captured, k)
        for x, y in zip(now, inputs[k]):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured.outputs(), want[k]):
            assert torch.equal(x, y), f"replay {k}"
        eager_again = _prefill_case(700 + k, fmt)
        _same_as_formula(eager_again, eager_again["call"]())


# ------------------------------------------------------------------ calls between each other

def _prefill_case(seed, fmt, rows=((3000, 3), (0, 40), (1500, 5))):
    """A call whose tiles are split (two launches and a workspace)."""
    g = _gen(seed)
    lens, new = [a + b for a, b in rows], [b for _, b in rows]
    held = [-(-x // PAGE) for x in lens]
    order = torch.randperm(sum(held), generator=g).to(torch.int32)
    table, live = torch.zeros(len(rows), max(held), dtype=torch.int32), torch.ones(sum(held), PAGE, dtype=torch.bool)
    k = 0
    for row, h in enumerate(held):
        table[row, :h] = order[k:k + h]
        k += h
    K, V = (torch.randn(sum(held), HKV, PAGE, D, generator=g) for _ in range(2))
    cache = C.cache_of(K, V, live, fmt, amax=torch.full((2 * HKV,), 4.0))
    cu = [0]
    for a in new:
        cu.append(cu[-1] + a)
    Q = torch.randn(cu[-1], HQ, D, generator=g).to(torch.bfloat16).cuda().transpose(0, 1)
    args = (rbs.make_shape(cu[-1], HQ, HKV, 64), Q, cache, table.cuda(), _ints(lens), _ints(cu))
    return dict(call=lambda **more: rbs.rbs_paged_prefill(*args, **more), Q=Q, cache=cache, table=table, lens=lens, new=new, cu=cu)


def _same_as_formula(c, O):
    K, V = C.cache_values(c["cache"])
    for row, (n, a) in enumerate(zip(c["lens"], c["new"])):
        at = slice(c["cu"][row], c["cu"][row + 1])
        keys, values = (R.gather(x, c["table"][row], n, PAGE) for x in (K, V))
        o, _, tol, _ = C.attend(c["Q"][:, at].cpu().double(), keys, values, SCALE, n - a + torch.arange(a), one_part=True)
        assert bool(((O[:, at].cpu().double() - o).abs() <= tol).all()), f"row {row}"


def test_captured_calls_side_by_side():
    """Two graphs captured on one stream, replayed at once on two: each has a workspace of its own."""
    cases = [_prefill_case(800, "bf16"), _prefill_case(801, "fp4", ((5000, 2), (700, 30)))]
    want = [c["call"]() for c in cases]
    for c, O in zip(cases, want):
        _same_as_formula(c, O)
    torch.cuda.synchronize()
    s, graphs, outs = torch.cuda.Stream(), [], []
    for c in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(c["call"]())
        graphs.append(graph)
    other = torch.cuda.Stream()
    for _ in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        between = cases[0]["call"]()
        torch.cuda.synchronize()
        for got, O in ((outs[0], want[0]), (outs[1], want[1]), (between, want[0])):
            assert torch.equal(got, O)


def test_threads_that_call_on_one_stream():
    """Calls of three threads, of two launches each, between each other."""
    cases = [_prefill_case(810 + k, FORMATS[k]) for k in range(3)]
    want = [c["call"]() for c in cases]
    torch.cuda.synchronize()
    got, failed = [[] for _ in cases], []

    def work(k):
        try:
            for _ in range(10):
                got[k].append(cases[k]["call"]())
        except Exception as e:  # noqa: BLE001 (told by the test)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for k in range(3):
        assert len(got[k]) == 10 and all(torch.equal(O, want[k]) for O in got[k])


# ------------------------------------------------------------------ streams given by name

def _memory_of(t):
    """Handle of the stream whose memory a tensor is."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not torch's memory")


@pytest.mark.parametrize("which", ["side", "default"])
def test_outputs_are_the_memory_of_the_calls_stream(which, monkeypatch):
    monkeypatch.setattr(P, "_workspaces", threading.local())
    c = _prefill_case(820, "fp4")
    read_shape = rbs.make_shape(c["lens"][0], HQ, HKV, 64)
    read_args = (read_shape, c["cache"], c["table"][:1].cuda(), _ints([0, c["lens"][0]]))
    x = torch.randn(2, HKV, 40, D, generator=_gen(821)).to(torch.bfloat16).cuda()
    slots = torch.arange(40, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    side, default = torch.cuda.Stream(), torch.cuda.default_stream()
    stream, here = (side, default) if which == "side" else (default, side)
    written = [C.make_cache(4, HKV, PAGE, "fp4") for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(here):
        O, (K, V) = c["call"](stream=stream), rbs.rbs_cache_read(*read_args, stream=stream)
        rbs.rbs_cache_write(rbs.make_shape(40, HQ, HKV, 64), x[0], x[1], written[0], slots, stream=stream)
        torch.cuda.synchronize()
        want, (K2, V2) = c["call"](), rbs.rbs_cache_read(*read_args)
        rbs.rbs_cache_write(rbs.make_shape(40, HQ, HKV, 64), x[0], x[1], written[1], slots)
    torch.cuda.synchronize()
    for t in (O, K, V):
        assert _memory_of(t) == stream.cuda_stream
    for t in (want, K2, V2):
        assert _memory_of(t) == here.cuda_stream
    assert torch.equal(O, want) and torch.equal(K, K2) and torch.equal(V, V2)
    for name in ("K", "V", "K_scale", "V_scale"):
        assert torch.equal(getattr(written[0], name), getattr(written[1], name))
    made = {key[1]: _memory_of(ws) for key, ws in P._workspaces.__dict__.items()}
    assert made[stream.cuda_stream] == stream.cuda_stream and made[here.cuda_stream] == here.cuda_stream


# ------------------------------------------------------------------ caches of two types

@pytest.mark.parametrize("to", FORMATS)
@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_moved_to_another_cache(fmt, to):
    """A row read from one cache and written to another of any type and page size: as that type holds the first one's values."""
    c = _prefill_case(830, fmt, ((0, 333),))
    n = 333
    K, V = rbs.rbs_cache_read(rbs.make_shape(n, HQ, HKV, 64), c["cache"], c["table"].cuda(), _ints([0, n]))
    amax = torch.full((2 * HKV,), 5.0).cuda() if to == "fp8" else None
    second = C.make_cache(6, HKV, 64, to, "tokens", amax)
    rbs.rbs_cache_write(rbs.make_shape(n, HQ, HKV, 64), K, V, second, torch.arange(n, dtype=torch.int32, device="cuda"))
    table = torch.arange(6, dtype=torch.int32)[None]
    K2, V2 = rbs.rbs_cache_read(rbs.make_shape(n, HQ, HKV, 64), second, table.cuda(), _ints([0, n]))
    for x, y in ((K, K2), (V, V2)):
        x, y = x.cpu(), y.cpu()
        if to == "bf16" or to == fmt == "fp4":
            assert torch.equal(x, y)  # (codes and powers of two come back as they were, the values at least)
        elif to == "fp4":
            assert torch.equal(C.e2m1_values(*C.e2m1_encode(x)), y.double())
        else:
            # Half a step of E4M3 (2^-4 of a normal value, 2^-10 of the units below 2^-6) and the roundings around it.
            unit = 5.0 / 448
            clamped = x.double().clamp(-5.0, 5.0)
            tol = (clamped.abs() * 2.0 ** -4).clamp(min=unit * 2.0 ** -10) * (1 + 2.0 ** -6) + clamped.abs() * 2.0 ** -8
            assert bool(((y.double() - clamped).abs() <= tol).all())


def test_debug_mode():
    """The calls drain their stream and report what failed: nothing here."""
    c = _prefill_case(840, "fp4")
    was = rbs.rbs_set_debug(True)
    try:
        O = c["call"]()
        assert torch.cuda.current_stream().query()
        K, V = rbs.rbs_cache_read(rbs.make_shape(50, HQ, HKV, 64), c["cache"], c["table"][:1].cuda(), _ints([0, 50]))
        assert torch.cuda.current_stream().query()
        rbs.rbs_cache_write(rbs.make_shape(50, HQ, HKV, 64), K, V, c["cache"], torch.arange(50, dtype=torch.int32, device="cuda") - 50)
    finally:
        rbs.rbs_set_debug(was)
    _same_as_formula(c, O)
