"""The testing hooks of distillation and the beams refuse what makes no sense (no GPU needed)."""


def test_lose_rows():
    from paper_2607_03011_gb300 import isoloco
    L = isoloco.lib()
    assert L.isoloco_debug_lose_rows(-1) == isoloco.ERR_INVALID and L.isoloco_debug_lose_rows(0) == isoloco.OK


def test_refuse_clusters():
    from paper_2607_03011_gb300 import isoloco
    L = isoloco.lib()
    for bad in (-1, 2):
        assert L.isoloco_debug_refuse_clusters(bad) == isoloco.ERR_INVALID
    assert L.isoloco_debug_refuse_clusters(0) == isoloco.OK
