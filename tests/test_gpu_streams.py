"""GPU: the outputs and workspaces that a call on a stream given by name makes itself."""

from __future__ import annotations

import pytest
import torch

import paper_2609_20971_amd as rbs
from paper_2609_20971_amd import _lib as L

pytestmark = pytest.mark.gpu

HQ, HKV, B, N, D = 4, 2, 64, 300, 128


def _memory_of(t):
    """Handle of the stream whose memory a tensor is."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not torch's memory")


def _tensors(x):
    if isinstance(x, torch.Tensor):
        return [x]
    if isinstance(x, tuple):
        return [t for y in x for t in _tensors(y)]
    return [t for t in vars(x).values() if isinstance(t, torch.Tensor)]


def _calls(stream):
    """Every call that makes outputs, each with tensors made ahead; (name, outputs)."""
    g = torch.Generator().manual_seed(4)
    Q, K, V = (torch.randn(h, N, D, generator=g).to(torch.bfloat16).cuda() for h in (HQ, HKV, HKV))
    shape, batch = rbs.make_shape(N, HQ, HKV, B), rbs.Batch([200, 100])
    vshape = rbs.varlen_shape(batch, HQ, HKV, B)
    stats, box, vstats = rbs.rbs_block_stats(shape, K), rbs.rbs_block_box(shape, K), rbs.rbs_block_stats_varlen(vshape, batch, K)
    lists, vlists = rbs.rbs_dense_indices(shape), rbs.rbs_dense_indices_varlen(vshape, batch)
    f8 = rbs.rbs_fp8_prepare(shape, Q, K, V)
    torch.cuda.synchronize()
    rules, s = (0.9, 0.95, 1, 2, 0), dict(stream=stream)
    yield "stats", rbs.rbs_block_stats(shape, K, **s)
    yield "box", rbs.rbs_block_box(shape, K, **s)
    yield "select", rbs.rbs_select(shape, Q, stats, *rules, **s)
    yield "variant", rbs.rbs_select_variant(shape, Q, stats, "box", 0.9, 1, 2, 0, box=box, **s)
    yield "prefill", rbs.rbs_sparse_prefill(shape, Q, K, V, *lists, **s)
    yield "fused", rbs.rbs_select_attend(shape, Q, K, V, stats, *rules, **s)
    yield "dense", rbs.rbs_dense_indices(shape, **s)
    yield "stats of a batch", rbs.rbs_block_stats_varlen(vshape, batch, K, **s)
    yield "select of a batch", rbs.rbs_select_varlen(vshape, batch, Q, vstats, *rules, **s)
    yield "prefill of a batch", rbs.rbs_sparse_prefill_varlen(vshape, batch, Q, K, V, *vlists, **s)
    yield "dense lists of a batch", rbs.rbs_dense_indices_varlen(vshape, batch, **s)
    yield "fp8 inputs", rbs.rbs_fp8_prepare(shape, Q, K, V, **s)
    yield "fp8 prefill", rbs.rbs_sparse_prefill_fp8(shape, f8, *lists, **s)


@pytest.mark.parametrize("which", ["side", "default"])
def test_outputs_are_the_memory_of_the_calls_stream(which, monkeypatch):
    monkeypatch.setattr(L, "_workspaces", {})
    side, default = torch.cuda.Stream(), torch.cuda.default_stream()
    stream, here = (side, default) if which == "side" else (default, side)
    with torch.cuda.stream(here):
        got = dict(_calls(stream))
        torch.cuda.synchronize()
        want = dict(_calls(None))
    torch.cuda.synchronize()
    for name, out in got.items():
        for t in _tensors(out):
            assert _memory_of(t) == stream.cuda_stream, name
        for t in _tensors(want[name]):
            assert _memory_of(t) == here.cuda_stream, name
    for name in ("prefill", "prefill of a batch", "fp8 prefill"):
        assert torch.equal(got[name], want[name]), name
    for name in ("select", "variant", "fused"):
        assert torch.equal(got[name][0], want[name][0]), name
    assert torch.equal(got["fused"][2], want["fused"][2])
    made = {k[1]: _memory_of(ws) for k, ws in L._workspaces.items()}
    assert made[stream.cuda_stream] == stream.cuda_stream and made[here.cuda_stream] == here.cuda_stream
