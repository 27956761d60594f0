"""Argument errors of the tree and eviction entry points that the host finds before
it touches CUDA."""
import os
import re

import pytest

NAMES = ("optr_tree_attention", "optr_tree_attention_win", "optr_verify_tree", "optr_kv_score",
         "optr_kv_score_win", "optr_evict_select",
         "optr_kv_compact", "optr_kv_compact_win")


@pytest.fixture(scope="module")
def lib():
    from paper_2608_02691_gb300 import build, optr
    build.build()
    return optr.lib()


@pytest.mark.parametrize("name", NAMES)
def test_null_handles(lib, name):
    from paper_2608_02691_gb300 import optr
    fn = getattr(lib, name)
    _, args = optr._SIG[name]
    assert fn(*[None if a is optr._V else 1 for a in args]) == -1


def test_flags_are_bits_of_their_own():
    from paper_2608_02691_gb300 import optr
    src = open(os.path.join(os.path.dirname(__file__), "..", "include", "optr.h")).read()
    bits = {n: int(v) for n, v in re.findall(r"#define (OPTR_DEVERR_\w+) (\d+)u", src)}
    for n in ("OPTR_DEVERR_TREE", "OPTR_DEVERR_KEPT"):
        assert bits[n] == getattr(optr, n)
    assert len(set(bits.values())) == len(bits) and all(v & (v - 1) == 0 for v in bits.values())
    assert int(re.search(r"OPTR_TREE_MAX_ROWS (\d+)", src)[1]) == optr.TREE_MAX_ROWS
