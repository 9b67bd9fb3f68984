"""A wait that gave up is reported, whatever other streams and threads do meanwhile."""
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean():
    from paper_2607_03011_gb300 import inner
    inner.status()
    yield
    inner.status()


def raise_on(stream):
    from paper_2607_03011_gb300 import isoloco
    assert isoloco.lib().isoloco_debug_raise_inner(stream.cuda_stream) == isoloco.OK


def test_reported_once_and_cleared():
    from paper_2607_03011_gb300 import inner, isoloco
    assert inner.status() == isoloco.OK
    s = torch.cuda.Stream()
    raise_on(s)
    s.synchronize()
    assert inner.status() == isoloco.ERR_TIMEOUT and isoloco.last_error()
    assert inner.status() == isoloco.OK
    raise_on(s)
    assert inner.status(stream=s) == isoloco.ERR_TIMEOUT and inner.status(stream=s) == isoloco.OK


def test_an_error_raised_while_another_thread_asks_is_not_lost():
    from paper_2607_03011_gb300 import inner, isoloco
    asked, raised = torch.cuda.Stream(), torch.cuda.Stream()
    seen, stop = [0], threading.Event()

    def ask():
        while not stop.is_set():
            if inner.status(stream=asked) == isoloco.ERR_TIMEOUT:
                seen[0] += 1

    th = threading.Thread(target=ask)
    th.start()
    try:
        for i in range(1000):
            before = seen[0]
            raise_on(raised)
            raised.synchronize()
            t0 = time.monotonic()
            while seen[0] == before and time.monotonic() - t0 < 1.0:
                time.sleep(0)
            assert seen[0] > before, f"the error raised in pass {i} was never reported"
    finally:
        stop.set()
        th.join()
