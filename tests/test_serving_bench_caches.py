"""The benchmark's serving mode with a cache in 4 bits and with more tokens behind the prompts."""

from __future__ import annotations

import json
import sys

import pytest

import bench


def test_one_type_of_cache(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["bench.py", "--serve", "2", "--serve-fp8", "--serve-fp4"])
    with pytest.raises(SystemExit) as e:
        bench.main()
    assert e.value.code == 2 and "not allowed with" in capsys.readouterr().err


@pytest.mark.gpu
@pytest.mark.parametrize("flags,cache", [(["--serve-fp4"], "fp4 e2m1"), (["--serve-fp8"], "fp8 e4m3"), ([], "bf16")])
def test_more_tokens_behind_the_prompts(flags, cache, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["bench.py", "--serve", "3", "--workload", "tiny-2k", "--steps", "4", "--serve-append", "70", *flags])
    bench.main()
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["mode"] == "serve" and line["rows"] == 3 and line["cache"] == cache and line["append_tokens"] == 70
    for name in ("append_norm_rope_ms", "append_attention_ms", "append_tflops", "decode_step_us", "decode_kv_gbps"):
        assert line[name] > 0, name


@pytest.mark.gpu
def test_four_bits_alone(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["bench.py", "--serve", "2", "--workload", "tiny-2k", "--steps", "3", "--serve-fp4"])
    bench.main()
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["cache"] == "fp4 e2m1" and "append_tokens" not in line and line["decode_step_us"] > 0
