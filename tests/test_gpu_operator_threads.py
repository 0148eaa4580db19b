"""Operators called from several host threads, each on a stream of its own."""
import threading

import pytest
import torch

from paper_2607_23115_gb300 import experts, fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _together(calls, turns):
    """Each call many times in a thread and on a stream of its own, against its first result."""
    want = [c() for c in calls]
    torch.cuda.synchronize()
    start, errors = threading.Barrier(len(calls)), []

    def work(call, want):
        try:
            stream = torch.cuda.Stream()
            differ = torch.zeros((), dtype=torch.int64, device=DEV)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                start.wait()
                for i in range(turns):
                    differ += (call() != want).sum()
                    if i % 50 == 49:
                        stream.synchronize()
            stream.synchronize()
            assert differ.item() == 0
        except BaseException as e:  # noqa: BLE001 - handed to the test's thread
            errors.append(e)
            start.abort()

    threads = [threading.Thread(target=work, args=a) for a in zip(calls, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_few_rows_of_different_lengths():
    """One kernel, whose shared memory goes by the length."""
    calls = []
    for k in (1024, 4096, 9000, 14000):
        torch.manual_seed(k)
        x = torch.randn(3, k, device=DEV).to(torch.bfloat16)
        w = fp8.quantize_weight(0.02 * torch.randn(512, k, device=DEV))
        calls.append(lambda x=x, w=w: fp8.linear(x, w))
    _together(calls, 3000)


def test_many_rows_and_experts():
    torch.manual_seed(0)
    calls = []
    for m, n, k in ((40, 4096, 1024), (300, 2000, 640), (2560, 2304, 512)):
        x = torch.randn(m, k, device=DEV).to(torch.bfloat16)
        w = fp8.quantize_weight(0.02 * torch.randn(n, k, device=DEV))
        calls.append(lambda x=x, w=w: fp8.linear(x, w))
    x = torch.randn(200, 512, device=DEV).to(torch.bfloat16)
    w = fp8.quantize_weight(0.02 * torch.randn(8, 384, 512, device=DEV))
    ids, g = torch.randint(0, 8, (200, 2), device=DEV), torch.rand(200, 2, device=DEV)

    def layer():
        plan = experts.sort(ids, 8)
        return experts.combine(experts.linear(x, plan, w), plan, g)

    calls.append(layer)
    _together(calls, 300)
