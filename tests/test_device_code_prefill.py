"""Properties of the paged prefill's gfx950 code, read from its disassembly (CPU only)."""

from __future__ import annotations

from tests.test_device_code import _functions, listing  # noqa: F401 (a fixture)


def test_the_join_has_no_rule_of_its_own(listing):  # noqa: F811
    """How tiles are divided is found once, by the first launch, in floating point: a second copy of the rule that rounds
    another way would leave tiles unjoined.  The rule's conversions of float to signed numbers mark it (divisions of
    whole numbers convert to unsigned ones)."""
    found = {True: 0, False: 0}
    for lines in listing:
        for name, code in _functions(lines):
            if "paged_prefill" in name:
                join = "join" in name
                marks = [x for _, x in code if x.startswith("v_cvt_i32_f32")]
                found[join] += 1
                assert bool(marks) != join, (name, marks[:3])
    assert found[True] >= 6 and found[False] >= 12
