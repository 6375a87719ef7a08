"""How the adapters' kernels give up, read from their source: every wait on a barrier in shared
memory is one of the bounded helper's, whose result is looked at and reported, and no block ends
while copies may be under way."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14618_gb300", "csrc")
TEXT = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "polyq_adapters_dev.cuh")).read())


def _kernel(name):
    start = TEXT.index(f" {name}(const __grid_constant__")
    return TEXT[start:TEXT.index("\n}\n", start)]


def test_waits_are_bounded_and_reported():
    assert not re.search(r"try_wait|test_wait|while \(!mbar", TEXT)
    body = _kernel("shrink_tiled_kernel")
    waits = re.findall(r"!mbar_wait\(", body)
    assert len(waits) == len(re.findall(r"mbar_wait\(", TEXT)) == 3
    assert len(re.findall(r"atomicExch\(P\.status, kStatusTimeout", body)) == 2


def test_blocks_stay_for_their_copies():
    """The warp that asks for stages waits for the last of them before it joins the others."""
    body = _kernel("shrink_tiled_kernel")
    asks = body.index("tma_load_3d")
    last = body.rindex("mbar_wait(full + 8 * (i % S::STAGES)")
    assert asks < last < body.index("__syncthreads();", last) < body.index("shrink_finish")
    for name in ("shrink_kernel", "gradients_kernel"):
        k = _kernel(name)
        assert k.rindex("cp_wait<0>()") > k.rindex("copy")
    assert "cp_wait<0>();\n}" in TEXT[TEXT.index("void expand_tile("):]
