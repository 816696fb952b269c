"""What asking for the device's status costs: one launch and one copy, however many kernels have a flag."""
import time

import pytest
import torch

import paper_2509_15763_b200 as ug

pytestmark = pytest.mark.gpu


def best(call, batches=10, calls=50):
    """Least time per call of several batches."""
    times = []
    for _ in range(batches):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(calls):
            call()
        times.append((time.perf_counter() - t) / calls)
    return min(times)


def test_a_status_costs_no_more_than_a_few_copies():
    """(A copy of each of the eight flags is ten times one copy; a launch and a copy about twice.)"""
    x = torch.zeros(1, device="cuda:0")
    ug.unigist_device_status(), x.item()
    assert best(ug.unigist_device_status) < 5 * best(lambda: x.item())


def test_threads_that_ask_at_once_report_a_timeout_once():
    """A wait that runs out (nothing faults and nothing hangs) while eight threads ask over and over: one of them hears of it."""
    import threading

    ug.unigist_device_status()
    for _ in range(2):
        heard, stop = [], threading.Event()

        def ask():
            while not stop.is_set():
                try:
                    ug.unigist_device_status()
                except ug.UnigistError as e:
                    heard.append(e.code)

        ug.unigist_selftest_wait_timeout()
        threads = [threading.Thread(target=ask) for _ in range(8)]
        for t in threads:
            t.start()
        torch.cuda.synchronize()
        time.sleep(0.2)
        stop.set()
        for t in threads:
            t.join()
        assert heard == [7]   # UNIGIST_ERR_TIMEOUT
        ug.unigist_device_status()
