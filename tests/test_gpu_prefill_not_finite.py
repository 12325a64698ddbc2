"""GPU: what is not finite in queries, attended keys and attended values reaches the results of attention over a paged
cache as the formula has it, however a row's keys are divided: among a workgroup's waves (rows of at most 32 queries),
in pieces that are joined, or not at all."""

from __future__ import annotations

import math

import pytest
import torch

from tests.test_gpu_prefill import D, _case, _run, _say

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "fp8", "fp4"]
# rows (cached before, new), heads.  Rows of at most 32 queries, whole and in pieces; of more, whole and in pieces.
FEW_WHOLE, FEW_SPLIT = ([(60, 4), (0, 3)], 8, 2), ([(6000, 3), (0, 2)], 8, 2)
MANY_WHOLE, MANY_SPLIT = ([(60, 90), (0, 3)], 8, 2), ([(6000, 40), (0, 3)], 8, 2)
KINDS = [FEW_WHOLE, FEW_SPLIT, MANY_WHOLE, MANY_SPLIT]


def _place(c, j):
    """Page and place in it of row 0's key j (a number or a tensor)."""
    page = c["table"][0].long()
    return (page[j // c["page"]], j % c["page"])


def _set(c, which, j, head, values, nan=False):
    """Row 0's key or value j of a head: all elements `values`, or one of them (5) NaN."""
    page, place = _place(c, j)
    t = getattr(c["cache"], which)
    if nan and c["fmt"] == "fp4":
        getattr(c["cache"], which + "_scale")[page, head, place, 0] = 255  # (its block of 32 elements)
    elif c["fmt"] == "bf16":
        t[page, head, place, 5 if nan else slice(None)] = math.nan if nan else values
    elif c["fmt"] == "fp8":
        t[page, head, place, 5 if nan else slice(None)] = 0x7F if nan else int(
            torch.tensor(values).to(torch.float8_e4m3fn).view(torch.uint8))
    else:  # +-1 (codes 2 and 10) times a power of two
        t[page, head, place] = 0x22 if values > 0 else 0xAA
        getattr(c["cache"], which + "_scale")[page, head, place] = 127 + int(math.log2(abs(values)))


def _elements(c):
    return slice(0, 32) if c["fmt"] == "fp4" else slice(5, 6)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", range(4))
def test_a_query_that_is_nan(kind, fmt):
    """Its result and its log-sum-exp are NaN (-inf is for tokens without keys); those beside it are as they were."""
    rows, hq, hkv = KINDS[kind]
    _say(f"[nan query] {rows} {fmt}")
    c = _case(rows, hq, hkv, 16, fmt, "heads", 70 + kind)
    clean, clean_lse = _run(c)
    c["q"][1, 5, 77] = math.nan
    O, lse = _run(c)
    assert bool(O[5, 1].isnan().all()) and bool(lse[5, 1].isnan())
    O[5, 1], lse[5, 1] = clean[5, 1], clean_lse[5, 1]
    assert torch.equal(O, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", range(4))
def test_keys_that_are_nan(kind, fmt):
    """Every second run of 32 keys: what attends one is NaN, its log-sum-exp too."""
    rows, hq, hkv = KINDS[kind]
    _say(f"[nan keys] {rows} {fmt}")
    c = _case(rows, hq, hkv, 16, fmt, "heads", 80 + kind)
    clean, clean_lse = _run(c)
    j = torch.arange(sum(rows[0]))
    _set(c, "K", j[j // 32 % 2 == 1], 1, 0.0, nan=True)
    O, lse = _run(c)
    new = rows[0][1]
    assert bool(O[4:, :new].isnan().all()) and bool(lse[4:, :new].isnan().all())
    assert torch.equal(O[:4], clean[:4]) and torch.equal(lse[:4], clean_lse[:4])
    assert torch.equal(O[:, new:], clean[:, new:]) and torch.equal(lse[:, new:], clean_lse[:, new:])


@pytest.mark.parametrize("fmt,low", [("bf16", -4.0), ("fp8", -4.0), ("fp4", -4.0), ("bf16", -math.inf)])
@pytest.mark.parametrize("kind", range(4))
def test_a_value_that_is_nan_of_a_small_weight(kind, fmt, low):
    """A NaN among attended values makes its element NaN, also where the weight rounds to 0 (logits of 512 for the first
    32 keys, -512 or -inf for the others); the other elements are the first 32 values' mean."""
    rows, hq, hkv = KINDS[kind]
    _say(f"[nan value] {rows} {fmt} {low}")
    c = _case(rows, hq, hkv, 16, fmt, "heads", 90 + kind)
    if fmt == "fp8":
        c["cache"].amax.fill_(448.0)
    before, new = rows[0]
    c["q"].fill_(1.0)
    j = torch.arange(before + new)
    for head in range(hkv):
        _set(c, "K", j[:32], head, 4.0)
        _set(c, "K", j[32:], head, low)
        _set(c, "V", j, head, 2.0)
    _set(c, "V", torch.tensor(before - 20), 1, 0.0, nan=True)
    O, lse = _run(c, 1.0)
    at = _elements(c)
    assert bool(O[4:, :new, at].isnan().all())
    O[4:, :new, at] = 2.0
    assert bool((O[:, :new] == 2.0).all())
    # The sum of 32 ones is exact; the logit and the change of base are a few steps of 515.
    assert bool(((lse[:, :new].cpu().double() - (512 + math.log(32))).abs() <= 515 * 8 * 2.0 ** -24).all())


@pytest.mark.parametrize("kind", range(4))
def test_logits_of_minus_infinity_alone(kind):
    """All keys of a token weigh nothing: the formula has 0 / 0, and zeros are for tokens without keys."""
    rows, hq, hkv = KINDS[kind]
    _say(f"[-inf] {rows}")
    c = _case(rows, hq, hkv, 16, "bf16", "heads", 60 + kind)
    clean, clean_lse = _run(c)
    before, new = rows[0]
    c["q"][:new] = 1.0
    _set(c, "K", torch.arange(before + new), 1, -math.inf)
    O, lse = _run(c)
    assert bool(O[4:, :new].isnan().all()) and bool((lse[4:, :new] == -math.inf).all())
    assert torch.equal(O[:, new:], clean[:, new:]) and torch.equal(lse[:, new:], clean_lse[:, new:])
    c["lens"] = [new - 1, rows[1][1]]  # the first token is before the row's first key
    O, lse = _run(c)
    assert bool((O[:, 0] == 0).all()) and bool((lse[:, 0] == -math.inf).all())
    assert bool(O[4:, 1:new].isnan().all())
