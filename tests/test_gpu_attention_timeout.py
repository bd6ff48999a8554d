"""A bounded wait of packed attention that runs out: recorded, reported once, and nothing else is disturbed.

No GPU is faulted or hung: the wait is that of a one-thread kernel without tensor memory or copies in flight and gives up
after a fraction of a millisecond, as the attention kernels' waits would after their one-second limit."""
import threading
import time

import pytest
import torch

from test_gpu_packed_attention import BF, backward, forward, make

pytestmark = pytest.mark.gpu
LIMIT = 200_000


def test_reported_once_and_calls_keep_their_results(cuda_device):
    import paper_1910_05124_b200 as pm
    op, q, k, v, d_o, cu = make([200, 77], 2, 1, 64, BF, cuda_device, seed=30)
    o, lse = forward(op, q, k, v, cu)
    g = backward(op, q, k, v, o, lse, d_o, cu)
    op.pm_attention_packed_status()
    op.pm_attention_packed_selftest_wait_timeout(LIMIT)
    op.pm_attention_packed_selftest_wait_timeout(LIMIT, stream=torch.cuda.Stream())      # one record for both
    torch.cuda.synchronize()
    o2, lse2 = forward(op, q, k, v, cu)
    g2 = backward(op, q, k, v, o, lse, d_o, cu)
    with pytest.raises(pm.PipeMareError, match="PM_ERR_TIMEOUT.*99"):
        op.pm_attention_packed_status()
    op.pm_attention_packed_status()
    o3, lse3 = forward(op, q, k, v, cu)
    for a, b, c in ((o, o2, o3), (lse, lse2, lse3), *((g[n], g2[n], g[n]) for n in g)):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_callers_at_the_same_time(cuda_device):
    """Of several callers that keep asking exactly one is told of each."""
    import paper_1910_05124_b200 as pm
    op = pm.PackedAttention(1, 1, 64)
    told, stop = [], threading.Event()

    def ask(stream):
        while not stop.is_set():
            try:
                op.pm_attention_packed_status(stream=stream)
            except pm.PipeMareError as e:
                told.append(str(e))
    threads = [threading.Thread(target=ask, args=(torch.cuda.Stream(),)) for _ in range(6)]
    probe = torch.cuda.Stream()
    for t in threads:
        t.start()
    try:
        for n in range(1, 201):
            op.pm_attention_packed_selftest_wait_timeout(LIMIT, stream=probe)
            probe.synchronize()
            deadline = time.monotonic() + 5.0
            while len(told) < n and time.monotonic() < deadline:
                time.sleep(0.0002)
            time.sleep(0.001)
            assert len(told) == n and "99" in told[-1], (n, len(told))
    finally:
        stop.set()
        for t in threads:
            t.join()


def test_limits_are_checked(cuda_device):
    import paper_1910_05124_b200 as pm
    op = pm.PackedAttention(1, 1, 64)
    for bad in (0, -1, 10 ** 9 + 1):
        with pytest.raises(pm.PipeMareError, match="limit_cycles"):
            op.pm_attention_packed_selftest_wait_timeout(bad)
