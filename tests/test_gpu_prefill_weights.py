"""GPU: the weights of rows of at most 32 queries (drafted tokens that are checked) have two bf16 parts, as those of the
decode calls, so that a token's result does not depend on which call gave it beyond the rounding of the result."""

from __future__ import annotations

import math

import pytest
import torch

import paper_2609_20971_amd as rbs
from tests import cache_reference as C
from tests import paged_reference as R
from tests.test_gpu_prefill import D, _case, _ints, _run, _say

pytestmark = pytest.mark.gpu

ROWS = [
    # rows (cached before, new), heads: whole, in pieces, among more rows than a wave has lanes
    ([(0, 4), (3, 1), (28, 4), (95, 3), (300, 2)], 8, 1),
    ([(6000, 3), (0, 4), (200, 8)], 8, 2),
    ([(2500, 32), (31, 1), (90, 5)], 4, 4),
    ([(9, None)] * 70 + [(3000, 4), (40, 2)], 28, 4),
]


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("k", range(len(ROWS)))
def test_few_queries(k, fmt):
    rows, hq, hkv = ROWS[k]
    _say(f"[weights] {rows[-3:]} {fmt}")
    c = _case(rows, hq, hkv, 16, fmt, "heads", 500 + k)
    O, lse = (x.cpu().double() for x in _run(c))
    O2 = _run(c, lse=False)[0].cpu().double()
    assert torch.equal(O, O2)
    K, V = C.cache_values(c["cache"])
    for row, (n, a) in enumerate(zip(c["lens"], c["new"])):
        if a == 0:
            continue
        at = slice(c["cu"][row], c["cu"][row + 1])
        k_, v_ = (R.gather(x, c["table"][row], n, 16) for x in (K, V))
        o, l, o_tol, l_tol = C.attend(c["q"][at].double().transpose(0, 1), k_, v_, 1 / math.sqrt(D), n - a + torch.arange(a))
        share = ((O[:, at] - o).abs() / o_tol)
        assert bool((share <= 1).all()), f"row {row} ({n - a} + {a}): {float(share.max()):.3f} of the tolerance"
        assert bool(((lse[:, at] - l).abs() <= l_tol).all()), f"row {row}: lse"


def test_single_tokens_are_decode_rows():
    """Two sums in different orders, each off by what the 64-bit comparison above allows it."""
    lens = [1, 17, 300, 1025, 4000]
    for fmt in ("bf16", "fp8", "fp4"):
        c = _case([(n - 1, 1) for n in lens], 16, 2, 16, fmt, "heads", 510)
        O, lse = _run(c)
        l2 = torch.empty_like(lse)
        O2 = rbs.rbs_paged_decode(rbs.make_shape(5, 16, 2, 64), c["q"].cuda().transpose(0, 1), c["cache"],
                                  c["table"].cuda(), _ints(lens), lse=l2)
        for row, n in enumerate(lens):
            k_, v_ = (R.gather(x, c["table"][row], n, 16) for x in C.cache_values(c["cache"]))
            _, _, o_tol, l_tol = C.attend(c["q"][row:row + 1].double().transpose(0, 1), k_, v_, 1 / math.sqrt(D),
                                          torch.tensor([n - 1]))
            at = slice(row, row + 1)
            assert bool(((O[:, at] - O2[:, at]).abs().cpu().double() <= 2 * o_tol).all()), (fmt, n)
            assert bool(((lse[:, at] - l2[:, at]).abs().cpu().double() <= 2 * l_tol).all()), (fmt, n)


@pytest.mark.parametrize("q", [0.0, 1.0])
@pytest.mark.parametrize("rows", [[(200, 4)], [(6000, 3)]])
def test_infinite_values_stay_infinite(rows, q):
    """In a block that is attended whole, where a weight is 1 (rest 0) and where rests have either sign after rounding."""
    c = _case(rows, 8, 1, 16, "bf16", "heads", 520)
    c["q"] *= q
    for j, sign, element in ((0, 1, 3), (37, -1, 9), (150, 1, 77)):
        c["cache"].V[int(c["table"][0, j // 16]), 0, j % 16, element] = sign * math.inf
    O, lse = _run(c)
    assert bool((O[:, :, [3, 77]] == math.inf).all()) and bool((O[:, :, 9] == -math.inf).all())
    O[:, :, [3, 9, 77]] = 0
    assert bool(O.isfinite().all()) and bool(lse.isfinite().all())
