"""Argument errors of the chunk, read-back and verification entry points that
the host finds before it touches CUDA."""
import os
import re

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2608_02691_gb300 import build, optr
    build.build()
    return optr.lib()


def test_null_handles(lib):
    assert lib.optr_chunk_workspace_size(None, 1, 1, 1) == 0
    assert lib.optr_chunk_attention(None, None, None, None, 1, None, None, 1, None, 1, 1, None, 1, None,
                                    None, 0, None) == -1
    assert lib.optr_chunk_attention_win(None, None, None, None, 1, None, None, 1, None, 1, 1, None, 1,
                                        None, None, 0, None, None, 0, None) == -1
    assert lib.optr_kv_read(None, 1, None, None, None, 1, 1, None, 1, None, None, None) == -1
    assert lib.optr_verify_drafts(None, None, None, 0, None, None, None, None, 1, 1, 1, None, None,
                                  None) == -1


def test_the_token_flag_is_a_bit_of_its_own():
    from paper_2608_02691_gb300 import optr
    src = open(os.path.join(os.path.dirname(__file__), "..", "include", "optr.h")).read()
    bits = {n: int(v) for n, v in re.findall(r"#define (OPTR_DEVERR_\w+) (\d+)u", src)}
    assert bits["OPTR_DEVERR_TOKEN"] == optr.OPTR_DEVERR_TOKEN
    assert len(set(bits.values())) == len(bits) and all(v & (v - 1) == 0 for v in bits.values())
