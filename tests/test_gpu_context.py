"""Contexts: what creating one costs, and that several threads can create theirs at once."""
import threading
import time

import pytest
import torch

from paper_2609_07883_b200 import binding as B
from paper_2609_07883_b200 import workloads as W

pytestmark = pytest.mark.gpu


def test_creating_a_context_does_not_ask_the_driver_for_what_it_knows():
    """The device's clock rates alone take the driver 2.4 ms.  (The quickest of many: the machine has other users.)"""
    shape, spent = W.AttnShape(32, 8, 128), []
    for _ in range(20):
        torch.cuda.synchronize()
        begin = time.perf_counter()
        ctx = B.Context(shape, 1000, 16, 4, 64)
        spent.append(time.perf_counter() - begin)
        ctx.close()
    assert min(spent) < 2e-3, f"{min(spent) * 1e3:.2f} ms"


def test_several_threads_create_contexts():
    shape, got = W.AttnShape(8, 2, 64), []

    def create():
        ctxs = [B.Context(shape, 100, 16, 4, 64) for _ in range(4)]
        got.append([B.sw_check_status(c) for c in ctxs])
        for c in ctxs:
            c.close()

    threads = [threading.Thread(target=create) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(got) == 4
