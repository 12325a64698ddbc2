"""Refusals of the calls over a paged cache, on the CPU: the C ABI's (nothing here
reaches a launch: each call fails validation first) and the binding's."""

from __future__ import annotations

import ctypes
import math

import pytest
import torch

import paper_2609_20971_amd as rbs

FAKE, MIS = 0x10000, 0x10008  # never dereferenced: validation fails before use
OK_PAST = 1                   # RBS_ERR_NULL of an argument checked after those in question


def _lib():
    return rbs.load()


def _pages(**over):
    v = dict(n_rows=4, max_pages=8, n_pages=20, page_size=16, page_table=FAKE, free_pages=FAKE)
    v.update(over)
    return rbs.rbs_pages(**v)


def _cache(**over):
    v = dict(n_pages=20, page_size=16, n_kv_heads=2, head_dim=128, format=0, stride_page=0, stride_head=0, stride_tok=0,
             K=FAKE, V=FAKE, amax=None)
    v.update(over)
    return rbs.rbs_cache(**v)


EXTEND = dict(seq_lens=FAKE, new_tokens=FAKE, n_free=FAKE, max_tokens=4, seq_lens_out=FAKE, n_free_out=FAKE,
              cu_tokens=FAKE, positions=FAKE, slots=FAKE, status=FAKE)


def _extend(pages, **over):
    a = dict(EXTEND, **over)
    return _lib().rbs_pages_extend(pages, *a.values(), None)


def _release(pages, **over):
    a = dict(dict(released=FAKE, seq_lens=FAKE, n_free=FAKE, status=FAKE), **over)
    return _lib().rbs_pages_release(pages, *a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(page_size=15), 3), (dict(page_size=8), 3), (dict(page_size=512), 3), (dict(page_size=48), 3),
    (dict(page_size=0), 3), (dict(page_size=-16), 3),
    (dict(n_rows=0), 2), (dict(n_rows=4097), 2), (dict(max_pages=0), 2), (dict(n_pages=0), 2), (dict(n_pages=-1), 2),
    (dict(max_pages=2**27, page_size=16), 2), (dict(n_pages=2**23, page_size=256), 2),
    (dict(page_table=None), 1), (dict(free_pages=None), 1), (dict(page_table=MIS), 5), (dict(free_pages=MIS), 5),
])
def test_pages_validation(over, code):
    assert _extend(_pages(**over)) == code
    assert _release(_pages(**over)) == code


def test_extend_and_release_arguments():
    assert _lib().rbs_pages_extend(None, *EXTEND.values(), None) == 1
    for name in EXTEND:
        if name == "max_tokens":
            continue
        if name != "new_tokens":
            assert _extend(_pages(), **{name: None}) == 1, name
        assert _extend(_pages(), **{name: MIS}) == 5, name
    for bad in (0, -1, (1 << 24) + 1):
        assert _extend(_pages(), max_tokens=bad) == 2
    for name in ("released", "seq_lens", "n_free", "status"):
        assert _release(_pages(), **{name: None}) == 1
        assert _release(_pages(), **{name: MIS}) == 5
    assert _release(None) == 1


CACHE_BAD = [
    (dict(page_size=8), 3), (dict(page_size=100), 3), (dict(head_dim=64), 3), (dict(format=2), 4), (dict(format=-1), 4),
    (dict(n_pages=0), 2), (dict(n_pages=2**23, page_size=256), 2), (dict(n_kv_heads=3), 2), (dict(n_kv_heads=0), 2),
    (dict(stride_tok=64), 2), (dict(stride_tok=136), 2), (dict(stride_head=-128), 2), (dict(stride_page=8), 2),
    (dict(stride_tok=2**22), 2), (dict(stride_page=2**60), 2),
    (dict(K=None), 1), (dict(V=None), 1), (dict(K=MIS), 5), (dict(V=MIS), 5),
    (dict(format=1), 1), (dict(format=1, amax=MIS), 5),
]


def _rope_c(**over):
    v = dict(q_weight=FAKE, k_weight=FAKE, inv_freq=FAKE, rot_dim=128, interleaved=0, eps=1e-6, factor=1.0)
    v.update(over)
    return rbs.rbs_rope(**v)


def _rope(shape=None, out=None, rope=None, cache=None, **over):
    shape = rbs.make_shape(10, 4, 2, 64) if shape is None else shape
    a = dict(Q=FAKE, K=FAKE, V=FAKE, positions=FAKE, Q_out=FAKE, K_out=FAKE)
    a.update({k: v for k, v in over.items() if k in a})
    return _lib().rbs_qk_norm_rope(shape, out, _rope_c() if rope is None else rope, *a.values(), cache,
                                   over.get("slots", FAKE), None)


def _decode(shape=None, cache=None, **over):
    shape = rbs.make_shape(10, 4, 2, 64) if shape is None else shape
    a = dict(Q=FAKE, page_table=FAKE, max_pages=4, seq_lens=FAKE, scale=0.0, O=FAKE, lse=FAKE, workspace=FAKE)
    a.update(over)
    return _lib().rbs_paged_decode(shape, _cache() if cache is None else cache, *a.values(), None)


@pytest.mark.parametrize("over,code", CACHE_BAD)
def test_cache_validation(over, code):
    assert _decode(cache=_cache(**over)) == code
    assert _rope(cache=_cache(**over)) == code


@pytest.mark.parametrize("field,value,code", [
    ("head_dim", 64, 3), ("n_tokens", 0, 2), ("n_q_heads", 3, 2), ("n_q_heads", 514, 2), ("n_kv_heads", 0, 2),
    ("q_stride_tok", 64, 2), ("q_stride_head", 4, 2),
])
def test_shapes(field, value, code):
    s = rbs.make_shape(10, 4, 2, 64)
    setattr(s, field, value)
    assert _decode(shape=s) == code
    assert _rope(shape=s) == code


def test_limits():
    assert _decode(shape=rbs.make_shape(4097, 4, 2, 64)) == 2
    assert _decode(shape=rbs.make_shape(4096, 4, 2, 64), Q=None) == OK_PAST
    assert _rope(shape=rbs.make_shape((1 << 24) + 1, 4, 2, 64)) == 2
    assert _rope(shape=rbs.make_shape(1 << 24, 4, 2, 64), Q=None) == OK_PAST
    assert _decode(max_pages=0) == 2 and _decode(max_pages=2**27) == 2
    assert _decode(shape=rbs.make_shape(4096, 4, 2, 64), max_pages=2**20) == 2   # 2^31 tiles of 32 keys
    assert _decode(shape=rbs.make_shape(4096, 4, 2, 64), max_pages=2**20 - 18, Q=None) == OK_PAST
    # Any block size, unlike the prefill's calls.
    assert _decode(shape=rbs.make_shape(10, 4, 2, 7), Q=None) == OK_PAST


def test_decode_arguments():
    assert _lib().rbs_paged_decode(rbs.make_shape(10, 4, 2, 64), None, FAKE, FAKE, 4, FAKE, 0.0, FAKE, None, FAKE, None) == 1
    for name in ("Q", "page_table", "seq_lens", "O", "workspace"):
        assert _decode(**{name: None}) == 1
    for name in ("Q", "page_table", "seq_lens", "O", "workspace", "lse"):
        assert _decode(**{name: MIS}) == 5
    for bad in (math.nan, math.inf):
        assert _decode(scale=bad) == 4
    assert rbs.rbs_decode_workspace_bytes() % 4 == 0


def test_rope_arguments():
    for name in ("Q", "K", "positions", "Q_out"):
        assert _rope(**{name: None}) == 1
    for name in ("Q", "K", "positions", "Q_out", "K_out"):
        assert _rope(**{name: MIS}) == 5
    for name in ("V", "slots"):
        assert _rope(cache=_cache(), **{name: None}) == 1
        assert _rope(cache=_cache(), **{name: MIS}) == 5
    for over, code in ((dict(rot_dim=-8), 3), (dict(rot_dim=136), 3), (dict(rot_dim=60), 3), (dict(eps=-1.0), 4),
                       (dict(eps=math.nan), 4), (dict(factor=math.inf), 4), (dict(inv_freq=None), 1),
                       (dict(inv_freq=MIS), 5), (dict(q_weight=MIS), 5), (dict(k_weight=MIS), 5)):
        assert _rope(rope=_rope_c(**over)) == code, over
    s, out = rbs.make_shape(10, 4, 2, 64), rbs.make_shape(10, 4, 2, 64)
    out.q_stride_head, out.q_stride_tok = 128, 4 * 128
    assert _rope(shape=s, out=out) == 2            # in place with other strides
    out = rbs.make_shape(11, 4, 2, 64)
    assert _rope(shape=s, out=out) == 2
    out = rbs.make_shape(10, 4, 2, 64)
    out.kv_stride_tok = 8
    assert _rope(shape=s, out=out) == 2


# ------------------------------------------------------------------ the binding

def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


@pytest.mark.parametrize("args,message", [
    ((_bf(4, 2, 16, 128), _bf(4, 2, 16, 128)), "must be on a GPU"),
    ((_bf(4, 2, 16, 128), _bf(4, 2, 16, 64)), "V must have shape"),
    ((_bf(4, 2, 16), _bf(4, 2, 16)), r"\[n_pages\]"),
    ((_bf(4, 2, 16, 128).float(), _bf(4, 2, 16, 128)), "must be torch.bfloat16"),
    ((_bf(4, 2, 16, 128), _bf(4, 2, 16, 128), torch.zeros(4)), "must be torch.uint8"),
    ((_bf(4, 2, 16, 128).byte(), _bf(4, 2, 16, 128).byte(), torch.zeros(3)), "amax must have shape"),
    ((_bf(4, 2, 16, 128), _bf(4, 16, 2, 128).transpose(1, 2)), "differ from K strides"),
    ((_bf(1, 2, 16, 128).expand(4, 2, 16, 128), _bf(1, 2, 16, 128).expand(4, 2, 16, 128)), "overlap"),
    ((_bf(0, 2, 16, 128), _bf(0, 2, 16, 128)), "overlap|holds none"),
])
def test_paged_cache_checks(args, message):
    with pytest.raises(ValueError, match=message):
        rbs.PagedCache(*args)


@pytest.mark.parametrize("over,message", [
    (dict(), "must be on a GPU"),
    (dict(page_table=_i32(4)), r"\[n_rows\]"),
    (dict(page_table=_i32(4, 5).long()), "must be torch.int32"),
    (dict(free_pages=_i32(4, 5)), "must have shape"),
    (dict(n_free=_i32(2)), "must have shape"),
    (dict(seq_lens=_i32(5)), "must have shape"),
    (dict(page_table=_i32(5, 4).t()), "must be contiguous"),
])
def test_pages_checks(over, message):
    a = dict(page_table=_i32(4, 5), free_pages=_i32(20), n_free=_i32(1), seq_lens=_i32(4))
    a.update(over)
    with pytest.raises(ValueError, match=message):
        rbs.Pages(*a.values(), 16)


def test_step_and_rope_checks():
    with pytest.raises(ValueError, match="cu_tokens must have shape"):
        rbs.PageStep(_i32(4), _i32(1), _i32(4), _i32(9), _i32(9), _i32(1))
    with pytest.raises(ValueError, match="slots must have shape"):
        rbs.PageStep(_i32(4), _i32(1), _i32(5), _i32(9), _i32(8), _i32(1))
    with pytest.raises(ValueError, match="must be on a GPU"):
        rbs.PageStep(_i32(4), _i32(1), _i32(5), _i32(9), _i32(9), _i32(1))
    with pytest.raises(ValueError, match="inv_freq must be torch.float32"):
        rbs.Rope(torch.zeros(64, dtype=torch.float64))
    with pytest.raises(ValueError, match="k_weight must have shape"):
        rbs.Rope(None, None, _bf(64))
    with pytest.raises(ValueError, match="must be on a GPU"):
        rbs.Rope(torch.zeros(64))
    for call in (lambda: rbs.rbs_pages_extend(object()), lambda: rbs.rbs_pages_release(object(), _i32(4))):
        with pytest.raises(ValueError, match="must be a Pages"):
            call()


def test_call_checks():
    shape = rbs.make_shape(10, 4, 2, 64)
    Q, K = _bf(4, 10, 128), _bf(2, 10, 128)
    rope = rbs.Rope(None)
    pos = _i32(10)
    for args, more, message in [
        ((Q, K, pos.long()), {}, "positions must be torch.int32"),
        ((Q, K, pos[:9]), {}, "positions must have shape"),
        ((Q[:3], K, pos), {}, "Q must have shape"),
        ((Q, K.float(), pos), {}, "K must be torch.bfloat16"),
        ((Q, K, pos), dict(Q_out=Q[:, :5]), "Q_out must have shape"),
        ((Q, K, pos), dict(K_out=K.float()), "K_out must be torch.bfloat16"),
        ((Q, K, pos), dict(cache=object()), "must be a PagedCache"),
        ((Q, K, pos), {}, "must be on a GPU"),
    ]:
        with pytest.raises(ValueError, match=message):
            rbs.rbs_qk_norm_rope(shape, rope, *args, **more)
    with pytest.raises(ValueError, match="must be a Rope"):
        rbs.rbs_qk_norm_rope(shape, object(), Q, K, pos)
    with pytest.raises(ValueError, match="must be a PagedCache"):
        rbs.rbs_paged_decode(shape, Q, object(), _i32(10, 3), pos)
    with pytest.raises(ValueError, match="Q must have shape"):
        rbs.rbs_paged_decode(shape, Q[:, :9], object(), _i32(10, 3), pos)


def test_rope_frequencies():
    f, factor = rbs.rope_frequencies(8, base=10000.0, device="cpu")
    assert factor == 1.0 and f.dtype == torch.float32
    assert torch.allclose(f.double(), torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-7)
    g, factor = rbs.rope_frequencies(8, base=10000.0, scaling="linear", scale=4.0, device="cpu")
    assert factor == 1.0 and torch.allclose(g, f / 4, rtol=1e-7)
    g, factor = rbs.rope_frequencies(128, scaling="parts", scale=4.0, device="cpu")
    full, _ = rbs.rope_frequencies(128, device="cpu")
    turns = 32768 * full.double() / (2 * math.pi)
    assert factor == pytest.approx(0.1 * math.log(4.0) + 1)
    # Whole turns decide; the interpolation runs over whole indices, so that pairs next to its ends are left out.
    assert torch.equal(g[turns > 45], full[turns > 45])
    assert torch.allclose(g[turns < 0.8], full[turns < 0.8] / 4, rtol=1e-6)
    ratio = (g / full).double()
    assert bool((ratio.diff() <= 1e-7).all()) and bool((ratio >= 0.25 - 1e-7).all())
    for bad in (dict(rot_dim=3), dict(base=1.0), dict(scale=0.5), dict(scaling="other"),
                dict(scaling="parts", fast=1.0, slow=2.0)):
        with pytest.raises(ValueError):
            rbs.rope_frequencies(**bad, device="cpu")


def test_threads_have_decode_workspaces_of_their_own(monkeypatch):
    """A call is two launches over the workspace: two threads' calls on one stream may interleave."""
    import threading

    from paper_2609_20971_amd import _paged
    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **dict(k, device="cpu")))
    got = {}

    def ask(name):
        got[name] = [_paged._workspace_of(0, 77), _paged._workspace_of(0, 77), _paged._workspace_of(0, 78)]

    threads = [threading.Thread(target=ask, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
        t.join()
    ask("here")
    for a, again, other in got.values():
        assert a is again and a is not other
        assert a.numel() * 4 >= rbs.rbs_decode_workspace_bytes()
    assert len({x.data_ptr() for three in got.values() for x in three}) == 2 * len(got)


# ------------------------------------------------------------------ packed queries

def _packed(shape=None, cache=None, **over):
    shape = rbs.make_shape(10, 4, 2, 64) if shape is None else shape
    a = dict(Q=FAKE, cu_tokens=FAKE, n_rows=5, page_table=FAKE, max_pages=4, seq_lens=FAKE, scale=0.0, O=FAKE, lse=FAKE,
             workspace=FAKE)
    a.update(over)
    return _lib().rbs_paged_decode_packed(shape, _cache() if cache is None else cache, *a.values(), None)


@pytest.mark.parametrize("over,code", CACHE_BAD)
def test_packed_cache_validation(over, code):
    assert _packed(cache=_cache(**over)) == code


def test_packed_arguments():
    for name in ("Q", "cu_tokens", "page_table", "seq_lens", "O", "workspace"):
        assert _packed(**{name: None}) == 1, name
    for name in ("Q", "cu_tokens", "page_table", "seq_lens", "O", "workspace", "lse"):
        assert _packed(**{name: MIS}) == 5, name
    for bad in (0, -1, 4097):
        assert _packed(n_rows=bad) == 2
    # More tokens than a table has rows, up to a step's; the tiles are counted over the rows.
    assert _packed(shape=rbs.make_shape(1 << 24, 4, 2, 64), n_rows=4096, Q=None) == OK_PAST
    assert _packed(shape=rbs.make_shape((1 << 24) + 1, 4, 2, 64)) == 2
    assert _packed(n_rows=4096, max_pages=2**20) == 2
    assert _packed(shape=rbs.make_shape(4096, 4, 2, 64), n_rows=1, max_pages=2**20, Q=None) == OK_PAST
    for bad in (math.nan, math.inf):
        assert _packed(scale=bad) == 4
    assert _lib().rbs_paged_decode_packed(None, _cache(), FAKE, FAKE, 5, FAKE, 4, FAKE, 0.0, FAKE, None, FAKE, None) == 1


def test_packed_binding_checks():
    shape = rbs.make_shape(10, 4, 2, 64)
    cache = object.__new__(rbs.PagedCache)
    object.__setattr__(cache, "device", -1)
    object.__setattr__(cache, "K", _bf(4, 2, 16, 128))
    table, lens, cu = _i32(6, 3), _i32(6), _i32(7)
    for t, s, c, message in [
        (table, lens, cu.long(), "cu_tokens must be torch.int32"),
        (table, lens, cu[:6], "cu_tokens must have shape"),
        (table, _i32(10), cu, "seq_lens must have shape"),
        (table, lens, None, "page_table must have shape"),
        (table, lens, cu, "must be on a GPU"),
    ]:
        with pytest.raises(ValueError, match=message):
            rbs.rbs_paged_decode(shape, _bf(4, 10, 128), cache, t, s, cu_tokens=c)


# ------------------------------------------------------------------ expanded tensors

def _expanded(h, n, over):
    """A bf16 [h][n][128] tensor that repeats its storage over the heads or over the tokens."""
    return (_bf(1, n, 128) if over == "heads" else _bf(h, 1, 128)).expand(h, n, 128)


@pytest.mark.parametrize("over", ["heads", "tokens"])
def test_expanded_tensors_are_refused(over):
    """Their stride of 0 would stand for the dense layout in the library, past the end of their storage."""
    shape, pos = rbs.make_shape(10, 4, 2, 64), _i32(10)
    Q, K, rope = _bf(4, 10, 128), _bf(2, 10, 128), rbs.Rope(None)
    cache = object.__new__(rbs.PagedCache)
    q, k = _expanded(4, 10, over), _expanded(2, 10, over)
    for args, more, name in [
        ((q, K, pos), {}, "Q"), ((Q, k, pos), {}, "K"), ((Q, k, pos), dict(V=k, cache=cache, slots=pos), "K"),
        ((Q, K, pos), dict(V=k, cache=cache, slots=pos), "V"), ((Q, K, pos), dict(Q_out=q), "Q_out"),
        ((Q, K, pos), dict(K_out=k), "K_out"),
    ]:
        with pytest.raises(ValueError, match=f"^{name} is expanded"):
            rbs.rbs_qk_norm_rope(shape, rope, *args, **more)
    for O in (None, q):
        with pytest.raises(ValueError, match="^Q is expanded"):
            rbs.rbs_paged_decode(shape, q, cache, _i32(10, 3), pos, O=O)
    with pytest.raises(ValueError, match="O strides"):
        rbs.rbs_paged_decode(shape, Q, cache, _i32(10, 3), pos, O=q)
    # The prefill's calls take their strides from the tensors as well.
    counts, indices = _i32(4, 1), _i32(4, 1)
    for args, name in [((q, K, K), "Q"), ((Q, k, k), "K"), ((Q, K, k), "V")]:
        with pytest.raises(ValueError, match=f"^{name} is expanded"):
            rbs.rbs_sparse_prefill(shape, *args, counts, indices, workspace=None)
    with pytest.raises(ValueError, match="^K is expanded"):
        rbs.rbs_block_stats(shape, k)


def test_one_head_or_token_may_have_any_stride():
    """(What it is stays unused: the checks after this one are reached.)"""
    shape = rbs.make_shape(1, 1, 1, 64)
    x = _bf(128).as_strided((1, 1, 128), (0, 0, 1))
    with pytest.raises(ValueError, match="must be on a GPU"):
        rbs.rbs_qk_norm_rope(shape, rbs.Rope(None), x, x, _i32(1))


def test_strides_over_one_head_or_token_need_not_agree():
    """K and V of one token (or KV head) from buffers of different layouts: only a missing GPU is left to refuse."""
    cache = object.__new__(rbs.PagedCache)
    for n, hkv, K, V, message in [
        (1, 2, _bf(2, 1, 128), _bf(1, 2 * 128 + 512)[:, :256].view(1, 2, 128).transpose(0, 1), "must be on a GPU"),
        (10, 1, _bf(1, 10, 128), _bf(3, 10, 128)[:1].as_strided((1, 10, 128), (7 * 1280, 128, 1)), "must be on a GPU"),
        (2, 2, _bf(2, 2, 128), _bf(2, 2, 128).transpose(0, 1), "differ from K strides"),
        (10, 1, _bf(1, 10, 128), _bf(10, 2, 128)[:, :1].transpose(0, 1), "differ from K strides"),
    ]:
        Q, pos = _bf(4, n, 128), _i32(n)
        object.__setattr__(cache, "device", -1)
        object.__setattr__(cache, "K", _bf(4, hkv, 16, 128))
        with pytest.raises(ValueError, match=message):
            rbs.rbs_qk_norm_rope(rbs.make_shape(n, 4, hkv, 64), rbs.Rope(None), Q, K, pos, V=V, cache=cache, slots=pos)
