"""Properties of the paged calls' gfx950 code, read from its disassembly (CPU only)."""

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


def test_rotation_into_other_formats_has_no_code_of_fp4(listing):  # noqa: F811
    """The packing of 4 bits takes registers that cost bf16 and FP8 callers waves: it is compiled apart."""
    apart = {True: 0, False: 0}
    for lines in listing:
        for name, code in _functions(lines):
            if "qk_norm_rope_kernel" in name:
                packs = any("_fp4_" in x.split()[0] for _, x in code)
                assert not (packs and any("_fp8_" in x.split()[0] for _, x in code)), name
                apart[packs] += 1
    assert apart[True] == apart[False] == 6
