"""Refusals of attention of prompts over a paged cache, on the CPU: the C ABI's (each
call fails validation before a launch) and the binding's."""

from __future__ import annotations

import math
import threading

import pytest
import torch

import paper_2609_20971_amd as rbs

FAKE, MIS = 0x10000, 0x10008  # never dereferenced: validation fails before use
NULL, SHAPE, UNSUPPORTED, ARG, ALIGN = 1, 2, 3, 4, 5


def _cache(**over):
    v = dict(n_pages=20, page_size=16, n_kv_heads=2, head_dim=128, format=0, stride_page=0, stride_head=0, stride_tok=0,
             K=FAKE, V=FAKE, amax=None)
    v.update(over)
    return rbs.rbs_cache(**v)


def _prefill(shape=None, cache=None, **over):
    a = dict(Q=FAKE, cu_tokens=FAKE, n_rows=5, page_table=FAKE, max_pages=4, seq_lens=FAKE, scale=0.0, O=FAKE, lse=FAKE,
             workspace=FAKE)
    a.update(over)
    return rbs.load().rbs_paged_prefill(rbs.make_shape(10, 4, 2, 64) if shape is None else shape,
                                        _cache() if cache is None else cache, *a.values(), None)


def test_arguments():
    for name in ("Q", "cu_tokens", "page_table", "seq_lens", "O", "workspace"):
        assert _prefill(**{name: None}) == NULL, name
    for name in ("Q", "cu_tokens", "page_table", "seq_lens", "O", "workspace", "lse"):
        assert _prefill(**{name: MIS}) == ALIGN, name
    for bad in (math.nan, math.inf, -math.inf):
        assert _prefill(scale=bad) == ARG
    for over in (dict(n_rows=0), dict(n_rows=-1), dict(n_rows=4097), dict(max_pages=0), dict(max_pages=1 << 27)):
        assert _prefill(**over) == SHAPE, over
    assert rbs.load().rbs_paged_prefill(None, _cache(), FAKE, FAKE, 5, FAKE, 4, FAKE, 0.0, FAKE, None, FAKE, None) == NULL
    assert rbs.load().rbs_paged_prefill(rbs.make_shape(10, 4, 2, 64), None, FAKE, FAKE, 5, FAKE, 4, FAKE, 0.0, FAKE, None, FAKE,
                                        None) == NULL
    assert rbs.rbs_prefill_workspace_bytes() % 16 == 0


def test_the_result_is_not_the_queries():
    assert _prefill(Q=FAKE, O=FAKE) == ARG


@pytest.mark.parametrize("over,code", [
    (dict(head_dim=64), UNSUPPORTED), (dict(n_tokens=0), SHAPE), (dict(n_tokens=(1 << 24) + 1), SHAPE),
    (dict(n_q_heads=3), SHAPE), (dict(n_q_heads=514), SHAPE), (dict(n_kv_heads=4), SHAPE), (dict(q_stride_tok=64), SHAPE),
    (dict(q_stride_head=100), SHAPE),
])
def test_shapes(over, code):
    s = rbs.make_shape(10, 4, 2, 64)
    for k, v in over.items():
        setattr(s, k, v)
    assert _prefill(shape=s) == code


@pytest.mark.parametrize("over,code", [
    (dict(page_size=24), UNSUPPORTED), (dict(format=2), ARG), (dict(format=1), NULL), (dict(format=4), NULL),
    (dict(format=4, K_scale=FAKE, V_scale=MIS), ALIGN), (dict(n_kv_heads=1), SHAPE), (dict(stride_tok=136), SHAPE),
    (dict(K=None), NULL), (dict(V=MIS), ALIGN),
])
def test_caches(over, code):
    assert _prefill(cache=_cache(**over)) == code


def test_largest_sizes_pass():
    assert _prefill(shape=rbs.make_shape(1 << 24, 64, 2, 64), n_rows=4096, max_pages=(1 << 27) - 1, Q=None) == NULL
    assert _prefill(shape=rbs.make_shape(1 << 24, 66, 2, 64)) == SHAPE


def test_binding_checks():
    shape = rbs.make_shape(10, 4, 2, 64)
    Q, i32 = torch.zeros(4, 10, 128, dtype=torch.bfloat16), lambda *s: torch.zeros(*s, dtype=torch.int32)
    for args, message in [((Q[:3], object(), i32(3, 4), i32(3), i32(4)), "Q must have shape"),
                          ((Q, object(), i32(3, 4), i32(3), i32(4)), "must be a PagedCache")]:
        with pytest.raises(ValueError, match=message):
            rbs.rbs_paged_prefill(shape, *args)


def test_workspaces_are_not_the_decode_calls(monkeypatch):
    """A thread's prefill and decode calls on a stream have workspaces of their own size, and threads of their own."""
    from paper_2609_20971_amd import _paged
    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **dict(k, device="cpu")))
    size = rbs.rbs_prefill_workspace_bytes
    got = []

    def ask():
        got.append([_paged._workspace_of(0, 5, size), _paged._workspace_of(0, 5, size), _paged._workspace_of(0, 5)])

    for _ in range(2):
        t = threading.Thread(target=ask)
        t.start()
        t.join()
    ask()
    for a, again, other in got:
        assert a is again and a is not other and a.numel() * 4 >= size()
    assert len({x.data_ptr() for g in got for x in g}) == 6
