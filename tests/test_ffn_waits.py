"""The waits of the gated block's pair kernel, read from its source (a wait that runs out cannot be
provoked in it without breaking the kernel)."""
import os
import re

from conftest import ROOT

SRC = re.sub(r"//[^\n]*", "", open(os.path.join(ROOT, "paper_2607_03011_gb300", "csrc", "ffn_gemm.cuh")).read())


def test_copies_in_flight_share_one_limit():
    assert "drain_barriers(" in SRC
    assert not re.search(r"\(void\)\s*mbar_wait\(&full", SRC)


def test_every_wait_that_gives_up_raises():
    waits = [m for m in re.finditer(r"(\(void\)\s*)?mbar_wait\(", SRC)]
    assert len(waits) >= 5
    for m in waits:
        if m[1]:
            assert SRC[m.end():].startswith("drain,"), "only the last wait, for MMAs already issued, has nobody to tell"
            continue
        after = SRC[m.end():m.end() + 260]
        assert "kErrTimeout" in after or "ok = false" in after, after


def test_no_tile_works_for_as_long_as_a_wait_may_last():
    """The weights' gradients sum over all tokens, up to 2^30 of them: 2^24 k-blocks, many seconds of work that is no
    failure.  A tile sums over a slice of them, so that its longest product is dx's, 2 ff, of 2^15 k-blocks."""
    depth = int(re.search(r"constexpr int kDepth = (\d+)", SRC)[1])
    tokens = int(re.search(r"constexpr int kSliceBlocks = (\d+) / kDepth;", SRC)[1])
    longest = max(tokens // depth, 2 * 2 ** 20 // depth)
    assert longest * 0.8e-6 < 0.1 * 2.0
    host = open(os.path.join(ROOT, "paper_2607_03011_gb300", "csrc", "ffn.cu")).read()
    assert re.search(r"kDw,[^;]*std::min\(planes \* kw, kSliceBlocks\)", host)
