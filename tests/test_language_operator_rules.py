"""Rules of the language operators that hold without a GPU: how memory is read, what host code refuses and asks for."""
import os
import re

import paper_2507_07149_b200 as daf

CSRC = os.path.join(os.path.dirname(daf.__file__), "csrc")


def test_lists_that_another_launch_writes_are_not_read_as_constant():
    # embedding_sum_kernel and embedding_join_kernel start while the sort still writes its list: read-only loads are for the caller's tokens
    with open(os.path.join(CSRC, "embedding.cu")) as f:
        loads = re.findall(r"__ldg\(([^;]*?)\s*\+", f.read())
    assert loads and all("a.tokens" in what for what in loads), loads
