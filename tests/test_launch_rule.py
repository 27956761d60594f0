"""Kernels are launched while the kernel before them may still run, so what that
one wrote is read past the non-coherent path: by __ldcg, bulk or asynchronous
copies.  A stale read cannot be provoked from a test; the sources are looked at."""
import os
import re

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2608_02691_gb300", "csrc")


def source(name):
    """The file without its comments."""
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_verification_reads_its_inputs_past_the_caches():
    src = source("verify.cu")
    for name in ("tp", "dp", "drafts", "u", "noise", "cu"):
        assert not re.search(rf"(?<![\w.]){name}\s*\[", src), name
        assert not re.search(rf"[(=?:,]\s*\*\s*{name}\b", src), name
    loads = re.findall(r"void load_vec\(.*?\n}", src, re.S)
    assert len(loads) == 2
    for body in loads:
        assert body.count("__ldcg(") == 2
        assert not re.search(r"[(=]\s*\*\s*(p\b|reinterpret_cast)", body)


def test_the_join_reads_what_the_attention_wrote_past_the_caches():
    src = source("chunk.cu")
    join = src[src.index("chunk_combine_kernel("):]
    join = join[:join.index("\n}\n")]
    assert "__ldcg(" in join
    for name in ("A.seg", "A.part", "A.cu", "A.pos0", "part", "from"):
        assert not re.search(rf"(?<![\w.&]){re.escape(name)}\s*\[", join), name
        assert not re.search(rf"[(=?:,]\s*\*\s*{re.escape(name)}\b", join), name
    assert not re.search(r"(?<!&)\bfrom->", join)
