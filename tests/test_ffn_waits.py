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


def test_the_wait_for_a_tile_grows_with_its_product():
    """A tile of dw_gate sums over all tokens, up to 2^30 of them: 2^24 k-blocks, many seconds of work that is no
    failure.  The epilogue's limit goes by the tile's k-blocks."""
    wait = re.search(r"mbar_wait\(&tfull\[buf\],([^{;]*)\)\)", SRC)
    assert wait and "q.kblocks" in wait[1], wait and wait[0]
