"""Refusals of the calls that move rows into a paged cache and out of it, and of
caches in 4 bits, on the CPU: the C ABI's (each call fails validation before a
launch) and the binding's."""

from __future__ import annotations

import pytest
import torch

import paper_2609_20971_amd as rbs

FAKE, MIS = 0x10000, 0x10008  # never dereferenced: validation fails before use
NULL, SHAPE, UNSUPPORTED, ARG, ALIGN = 1, 2, 3, 4, 5


def _cache(**over):
    v = dict(n_pages=20, page_size=16, n_kv_heads=2, head_dim=128, format=4, stride_page=0, stride_head=0, stride_tok=0,
             K=FAKE, V=FAKE, amax=None, K_scale=FAKE, V_scale=FAKE)
    v.update(over)
    return rbs.rbs_cache(**v)


def _write(shape=None, v_shape=None, cache=None, **over):
    a = dict(K=FAKE, V=FAKE)
    a.update({k: v for k, v in over.items() if k in a})
    return rbs.load().rbs_cache_write(rbs.make_shape(10, 4, 2, 64) if shape is None else shape, v_shape, *a.values(),
                                      _cache() if cache is None else cache, over.get("slots", FAKE), None)


def _read(shape=None, cache=None, **over):
    a = dict(cu_tokens=FAKE, starts=FAKE, n_rows=3, page_table=FAKE, max_pages=4, K=FAKE, V=FAKE)
    a.update(over)
    return rbs.load().rbs_cache_read(rbs.make_shape(10, 4, 2, 64) if shape is None else shape,
                                     _cache() if cache is None else cache, *a.values(), None)


def _decode(cache):
    return rbs.load().rbs_paged_decode(rbs.make_shape(10, 4, 2, 64), cache, FAKE, FAKE, 4, FAKE, 0.0, FAKE, None, FAKE, None)


def _rope(cache):
    rope = rbs.rbs_rope(q_weight=FAKE, k_weight=FAKE, inv_freq=FAKE, rot_dim=128, interleaved=0, eps=1e-6, factor=1.0)
    return rbs.load().rbs_qk_norm_rope(rbs.make_shape(10, 4, 2, 64), None, rope, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, cache,
                                       FAKE, None)


@pytest.mark.parametrize("over,code", [
    (dict(format=2), ARG), (dict(format=3), ARG), (dict(format=5), ARG),
    (dict(K_scale=None), NULL), (dict(V_scale=None), NULL), (dict(K_scale=MIS), ALIGN), (dict(V_scale=MIS), ALIGN),
    (dict(K=MIS), ALIGN), (dict(V=None), NULL), (dict(page_size=24), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
    (dict(stride_tok=144), SHAPE), (dict(stride_head=2048 + 64), SHAPE), (dict(stride_page=4096 + 16), SHAPE),
    (dict(stride_tok=64), SHAPE), (dict(n_kv_heads=3), SHAPE), (dict(n_pages=0), SHAPE),
])
def test_caches_in_4_bits(over, code):
    c = _cache(**over)
    assert [f(cache=c) for f in (_write, _read)] + [_decode(c), _rope(c)] == [code] * 4


def test_scales_are_not_read_of_other_formats():
    for c in (_cache(format=0, K_scale=None, V_scale=MIS, K=None), _cache(format=1, amax=FAKE, K_scale=MIS, V_scale=None, K=None)):
        assert _write(cache=c) == NULL  # K, and not the scales


def test_write_arguments():
    for name in ("K", "V", "slots"):
        assert _write(**{name: None}) == NULL, name
        assert _write(**{name: MIS}) == ALIGN, name
    assert rbs.load().rbs_cache_write(None, None, FAKE, FAKE, _cache(), FAKE, None) == NULL
    assert rbs.load().rbs_cache_write(rbs.make_shape(10, 4, 2, 64), None, FAKE, FAKE, None, FAKE, None) == NULL
    for over, code in ((dict(n_tokens=0), SHAPE), (dict(n_tokens=(1 << 24) + 1), SHAPE), (dict(head_dim=64), UNSUPPORTED),
                       (dict(n_kv_heads=4), SHAPE), (dict(n_q_heads=3), SHAPE), (dict(kv_stride_tok=64), SHAPE),
                       (dict(kv_stride_head=100), SHAPE)):
        s = rbs.make_shape(10, 4, 2, 64)
        for k, v in over.items():
            setattr(s, k, v)
        assert _write(shape=s) == code, over
        if "head_dim" not in over and "n_q_heads" not in over:
            assert _write(v_shape=s) == (NULL if "x" in over else SHAPE), over
    assert _write(shape=rbs.make_shape(1 << 24, 4, 2, 64), K=None) == NULL


def test_read_arguments():
    for name in ("cu_tokens", "page_table", "K", "V"):
        assert _read(**{name: None}) == NULL, name
    for name in ("cu_tokens", "starts", "page_table", "K", "V"):
        assert _read(**{name: MIS}) == ALIGN, name
    assert _read(starts=None, K=None) == NULL
    for over in (dict(n_rows=0), dict(n_rows=4097), dict(max_pages=0), dict(max_pages=1 << 27)):
        assert _read(**over) == SHAPE, over
    s = rbs.make_shape(10, 4, 2, 64)
    s.kv_stride_tok = 8
    assert _read(shape=s) == SHAPE
    assert _read(shape=rbs.make_shape((1 << 24) + 1, 4, 2, 64)) == SHAPE
    assert _read(cache=_cache(n_kv_heads=1)) == SHAPE


# ------------------------------------------------------------------ the binding

def _u8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def _bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


K4, S4 = (4, 2, 16, 64), (4, 2, 16, 4)


@pytest.mark.parametrize("args,message", [
    ((_u8(*K4), _u8(*K4), None, _u8(*S4), _u8(*S4)), "must be on a GPU"),
    ((_u8(*K4), _u8(*K4), torch.zeros(4), _u8(*S4), _u8(*S4)), "not both"),
    ((_u8(*K4), _u8(*K4), None, _u8(*S4)), "V_scale must be a torch.Tensor"),
    ((_u8(*K4), _u8(*K4), None, None, _u8(*S4)), "K_scale must be a torch.Tensor"),
    ((_bf(*K4), _bf(*K4), None, _u8(*S4), _u8(*S4)), "K must be torch.uint8"),
    ((_u8(*K4), _u8(*K4), None, _u8(*S4).float(), _u8(*S4)), "K_scale must be torch.uint8"),
    ((_u8(*K4), _u8(*K4), None, _u8(4, 2, 16, 8), _u8(*S4)), "K_scale must have shape"),
    ((_u8(*K4), _u8(*K4), None, _u8(4, 16, 2, 4).transpose(1, 2), _u8(*S4)), "are not 1/16"),
    ((_u8(1, 2, 16, 64).expand(*K4), _u8(1, 2, 16, 64).expand(*K4), None, _u8(*S4), _u8(*S4)), "overlap"),
])
def test_paged_cache_checks(args, message):
    with pytest.raises(ValueError, match=message):
        rbs.PagedCache(*args)


def test_allocate_takes_one_format():
    with pytest.raises(ValueError, match="not both"):
        rbs.PagedCache.allocate(4, 16, 2, amax=torch.zeros(4), device="cpu", fp4=True)


def test_call_checks():
    shape = rbs.make_shape(10, 4, 2, 64)
    K, slots = _bf(2, 10, 128), _i32(10)
    for args, message in [((K.float(), K, object(), slots), "K must be torch.bfloat16"),
                          ((K, K[:, :9], object(), slots), "V must have shape"),
                          ((K, K[:, :1].expand(2, 10, 128), object(), slots), "V is expanded"),
                          ((K, K, object(), slots), "must be a PagedCache")]:
        with pytest.raises(ValueError, match=message):
            rbs.rbs_cache_write(shape, *args)
    with pytest.raises(ValueError, match="must be a PagedCache"):
        rbs.rbs_cache_read(shape, object(), _i32(3, 4), _i32(4))
