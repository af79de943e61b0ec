"""The workspace of the layer for a few tokens is laid out once a call, by the check of its size, and what was checked is what the kernels use; what one of its
workgroups writes another reads in a later kernel only (read from the sources; no GPU)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1705_01598_amd", "csrc")


def test_the_layout_that_was_checked_is_the_one_that_is_used():
    calls = {}
    for path in glob.glob(os.path.join(CSRC, "*.*")):
        if path.endswith((".hpp", ".hip", ".cpp")):
            n = len(re.findall(r"\b(?:few_room|few_shares)\(", open(path).read()))
            if n:
                calls[os.path.basename(path)] = n
    # the definitions and one call of few_shares; the query and the call's check
    assert calls == {"decode.hpp": 3, "decode_api.cpp": 2}
    api = open(os.path.join(CSRC, "decode_api.cpp")).read()
    assert "workspace_bytes < room.bytes" in api and "a.room = room" in api


def test_no_workgroup_reads_what_another_of_its_kernel_wrote():
    """Shares of results go from kernel to kernel: no counters, and no stores that would have to be seen while their kernel runs."""
    for name in ("few.hpp", "few_layer.hpp"):
        text = open(os.path.join(CSRC, name)).read()
        assert not re.search(r"__hip_atomic|__MEMORY_SCOPE|\basm\b|__threadfence|amdgcn_fence", text), name
    assert re.findall(r"\batomic\w+\(([^,]+),", text) == ["&n.mask[2 * e + t / 32]"]      # LDS
