"""The waits and barriers of the distillation kernels, read from their source (a wait that runs out, or a barrier that
misses a warp, cannot be provoked in them without breaking the kernel)."""
import os
import re

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2607_03011_gb300", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_a_wait_that_gives_up_raises_and_waits_for_its_copy_once_more():
    src = source("distill.cu")
    waits = list(re.finditer(r"mbar_wait\(", src))
    assert len(waits) == 1
    after = src[waits[0].end():waits[0].end() + 300]
    assert "kErrTimeout" in after and "drain_barriers(" in after


def test_nobody_waits_for_a_barrier_that_is_not_set_up():
    src = source("distill.cu")
    init = src.index("mbar_init(&bar")
    assert init < src.index("__syncthreads();", init) < src.index("wait_row()", init)


def test_launches_bring_the_list_warp():
    """The kernels' barriers count THREADS + 32 threads."""
    src = source("distill.cu")
    assert set(re.findall(r"kAll = ([^;]+);", src)) == {"THREADS + 32"}
    assert re.findall(r"cfg\.blockDim = dim3\(([^)]+)\);", src) == ["THREADS + 32"] * 2
    assert len(re.findall(r"__launch_bounds__\(THREADS \+ 32,", src)) == 2


def test_warps_reach_collective_operations_whole():
    """No collective operation over a whole warp behind a condition that only some of its lanes meet."""
    for name in ("distill.cu", "beam.cu"):
        assert not re.search(r"(&&|\|\||\?)[^;?:]*__(reduce|shfl|ballot|any|all)\w*_sync\(", source(name)), name
