"""Where the product kernels bring a warp's lanes together, read from their
source: tcgen05's loads, stores and deallocation are instructions of the whole
warp, and lanes that gave up a wait alone would leave the others at the next
__syncwarp."""
import os
import re

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2607_14618_gb300", "csrc", "polyq_mm.cu")
TEXT = open(SRC).read()


def _kernel(name):
    start = TEXT.index(f"{name}(const __grid_constant__")
    return TEXT[start:TEXT.index("\n}\n", start)]


def _epilogue():
    body = _kernel("mm_pair")
    return body[body.index("epilogue: a lane owns a row"):]


def test_a_warp_gives_up_as_a_whole():
    """Every lane's wait decides for all lanes; no lane asks the flag alone."""
    e = _epilogue()
    loop = re.search(r"for \(int tc = 0; (.*?); \+\+tc\)", e).group(1)
    assert "s_abort" not in re.sub(r"__any_sync\(0xffffffffu, s_abort\)", "", loop)
    wait = e.index("wait(smem_u32(&bar_accf[buf])")
    assert re.match(r"[^\n]*\n\s*if \(!__all_sync\(0xffffffffu, w == kOk\)\) \{", e[wait:])


def test_lanes_are_together_before_a_chunk_is_loaded():
    """A chunk's outputs, and the residual of the next, are by lanes with a row."""
    assert re.search(r"__syncwarp\(\);[^\n]*\n\s*uint32_t r0\[32\][^\n]*\n\s*load\(c, r0, r1\);", _epilogue())


@pytest.mark.parametrize("kernel", ["mm_pair", "mm_few"])
def test_lanes_are_together_before_the_release(kernel):
    assert re.search(r"__syncwarp\(\);\s*tc_fence_after\(\);\s*tmem_dealloc", _kernel(kernel))


def test_the_few_kernel_loads_together():
    body = _kernel("mm_few")
    assert re.search(r"__syncthreads\(\);[^\n]*\n\s*__syncwarp\(\);\s*tc_fence_after\(\);", body)
