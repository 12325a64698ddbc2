"""GPU: the benchmark's serving mode, a prompt's path and captured decode steps, at a small size."""

from __future__ import annotations

import json
import sys

import pytest

import bench

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "fp8 e4m3"])
def test_serving_mode_prints_its_line(cache, monkeypatch, capsys):
    argv = ["bench.py", "--serve", "3", "--workload", "tiny-2k", "--steps", "4"]
    monkeypatch.setattr(sys, "argv", argv + (["--serve-fp8"] if cache != "bf16" else []))
    bench.main()
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["mode"] == "serve" and line["workload"] == "tiny-2k" and line["data"] == "synthetic"
    assert line["rows"] == 3 and line["steps"] == 4 and line["cache"] == cache
    for name in ("prompt_pages_ms", "prompt_norm_rope_ms", "prompt_prefill_ms", "decode_step_us", "decode_kv_gbps",
                 "decode_tokens_per_s"):
        assert line[name] > 0, name
