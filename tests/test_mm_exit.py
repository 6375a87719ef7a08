"""How the product kernels give up, read from their source: every wait of a role
has a limit, one that runs out raises the flag in both CTAs of a pair and sets
the status before anything else, and no CTA leaves while copies or arrivals may
still be on their way into its shared memory."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14618_gb300", "csrc")
MM = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "polyq_mm.cu")).read())
TC = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "polyq_tc.cuh")).read())


def _kernel(name):
    start = MM.index(f"{name}(const __grid_constant__")
    return MM[start:MM.index("\n}\n", start)]


def test_waits_are_bounded():
    """The kernels wait on barriers through two helpers only, and both count."""
    assert not re.search(r"try_wait|test_wait|mbar_try_wait", MM)
    for name in ("wait", "wait_stay"):
        body = re.search(rf"__forceinline__ \w+ {name}\(.*?\n}}\n", TC, re.S).group(0)
        assert "it < kSleepLimit" in body and "while" not in body
    limit = int(re.search(r"kSleepLimit = 1u << (\d+)", TC).group(1))
    ns = int(re.search(r"kSleepNs = (\d+)", TC).group(1))
    assert (1 << limit) * ns * 1e-9 < 10  # seconds


@pytest.mark.parametrize("kernel", ["mm_pair", "mm_few"])
def test_a_wait_that_runs_out_is_reported(kernel):
    """Each result of wait() is looked at, and a timeout goes to fail()."""
    body = _kernel(kernel)
    calls = len(re.findall(r"(?<![_\w])wait\(smem_u32", body))
    kept = len(re.findall(r"\bw = wait\(smem_u32", body))
    assert calls == kept > 0
    assert len(re.findall(r"if \(w == kTimeout\) fail\(", body)) >= 3
    fail = re.search(r"auto fail = .*?\n  };", body, re.S).group(0)
    assert fail.index("s_abort = 1") < fail.index("atomicExch(P.status") < fail.index("kStayCycles")
    if kernel == "mm_pair":  # the peer's flag too
        assert fail.index("mapa(") < fail.index("st.relaxed.cluster") < fail.index("atomicExch(P.status")


def test_a_give_up_outlasts_copies():
    """A millisecond or so of cycles: a thousand times a copy's time."""
    shift = int(re.search(r"kStayCycles = 1 << (\d+)", TC).group(1))
    assert 0.5e-3 < (1 << shift) / 2.07e9 < 5e-3


@pytest.mark.parametrize("kernel,barrier", [("mm_pair", "bar_done"), ("mm_few", "bar_acc")])
def test_ctas_stay_for_the_last_commit(kernel, barrier):
    """The issuer's last commit is on a barrier that it waits for, after any way
    out of its loop; of a pair the second CTA, where the commit arrives too, waits
    for it as well."""
    body = _kernel(kernel)
    issuer = body[body.index("elect_one", body.index("warp == 1")):body.index("__syncthreads();", body.index("copy_scales"))]
    commits = re.findall(r"commit<\d>\(smem_u32\(&(\w+)", issuer)
    assert commits[-1] == barrier
    assert len(re.findall(rf"wait_stay\(smem_u32\(&{barrier}\), 0\)", body)) == (2 if kernel == "mm_pair" else 1)


@pytest.mark.parametrize("kernel", ["mm_pair", "mm_few"])
def test_clusters_leave_together(kernel):
    """All roles meet before the tensor memory goes, and a cluster's CTAs before
    the first of them leaves."""
    end = _kernel(kernel)
    end = end[end.rindex("__syncthreads();"):]
    assert "cluster_sync();" in end and "tmem_dealloc" in end
