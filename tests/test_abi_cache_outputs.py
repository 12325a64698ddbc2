"""Refusals of outputs that would be written over each other, on the CPU (each call fails validation before a launch)."""

from __future__ import annotations

import paper_2609_20971_amd as rbs

FAKE, OTHER, MIS = 0x10000, 0x20000, 0x10008  # never dereferenced: validation fails before use
NULL, ARG, ALIGN = 1, 4, 5


def _read(K, V, page_table=FAKE):
    cache = rbs.rbs_cache(20, 16, 2, 128, 0, 0, 0, 0, FAKE, FAKE, None)
    return rbs.load().rbs_cache_read(rbs.make_shape(10, 4, 2, 64), cache, FAKE, None, 5, page_table, 4, K, V, None)


def test_keys_and_values_read_are_not_one_buffer():
    assert _read(FAKE, FAKE) == ARG
    assert _read(FAKE, FAKE, page_table=None) == NULL and _read(MIS, MIS) == ALIGN
    assert _read(FAKE, OTHER, page_table=MIS) == ALIGN  # (two buffers get as far as the next check)
