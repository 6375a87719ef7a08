"""A full host memory does not end the process in the device entry points: what
they cache is allocated under a handler (read from the source)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14618_gb300", "csrc")


@pytest.mark.parametrize("name", ["polyq_runtime.cu", "polyq_fp4.cu", "polyq_mm.cu"])
def test_containers_grow_under_a_handler(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    grows = [m.start() for m in re.finditer(r"\.emplace\(|\.insert\(|\.push_back\(|\bnew \w|std::vector<|g_\w+\[", text)]
    for at in grows:
        assert re.search(r"try \{\s*\w+$", text[:at]), text[at - 40:at + 40]
