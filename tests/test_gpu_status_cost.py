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
