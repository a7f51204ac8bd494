"""The transformer-block calls let other Python threads run while a launch waits for room in the device's queue."""
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


def test_other_threads_run_while_a_launch_waits(dp):
    """A stream that is busy for about a second takes about a thousand launches and lets the next wait; meanwhile this thread counts."""
    x = torch.randn((2, 2, 2, 16), device="cuda")
    y = torch.empty_like(x)
    stream = torch.cuda.Stream()
    call = lambda: dp.dpclip_qknorm_forward(x, None, None, None, None, y, None, stream=stream)            # noqa: E731
    call()
    torch.cuda.synchronize()
    clock = 1.5e9                                                   # cycles: a second at most
    ready = threading.Event()

    def launches():
        ready.wait()
        for _ in range(4000):
            call()

    t = threading.Thread(target=launches)
    t.start()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(int(clock))
    start = last = time.perf_counter()
    ready.set()
    gap = 0.0
    while t.is_alive():
        time.sleep(0.001)
        now = time.perf_counter()
        gap, last = max(gap, now - last), now
    t.join()
    torch.cuda.synchronize()
    waited = time.perf_counter() - start
    assert waited > 0.5, "the launches did not have to wait: nothing was tested"
    assert gap < 0.3, f"this thread stood still for {gap:.2f} s"
