"""Device helpers of the headers that no kernel calls are not kept: such a form
of an instruction would be compiled by nothing and run by no test."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14618_gb300", "csrc")
TEXT = "".join(re.sub(r"//[^\n]*", "", open(f).read()) for f in sorted(glob.glob(os.path.join(CSRC, "*"))))


@pytest.mark.parametrize("header", sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "*.cuh"))))
def test_every_helper_has_a_caller(header):
    text = open(os.path.join(CSRC, header)).read()
    names = set(re.findall(r"__(?:forceinline|inline)__[\w\s:*&<>]*?\b(\w+)\s*\(", text))
    alone = sorted(n for n in names if len(re.findall(rf"\b{n}\b", TEXT)) < 2)
    assert not alone
