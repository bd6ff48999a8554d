"""Packed attention over more sequences than one round of the tile search takes, empty ones among them."""
import random

import pytest
import torch

import operators_reference as R
from test_gpu_packed_attention import BF, F, check, forward, backward, make, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 40, 128])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [256, 257, 1024, 1025, 1100])
def test_short_and_empty_sequences(cuda_device, n, dtype, D):
    rng = random.Random(n + D)
    lens = [rng.choice([0, 0, 1, 2, rng.randint(0, 9), rng.randint(0, 40)]) for _ in range(n)]
    lens[rng.randrange(n)], lens[-1] = 300, rng.choice([0, 129])
    check(*make(lens, 1, 1, D, dtype, cuda_device, first=rng.choice([0, 3]), tail=rng.choice([0, 5]), seed=n))


@pytest.mark.parametrize("dtype", [BF, F])
def test_room_for_many_more_sequences(cuda_device, dtype):
    """A cu_seqlens of fixed size, nearly all of it empty sequences: right, and within a time that does not grow with its square
    (0.7 ms for the forward pass in bf16; a walk through all sequences in every block takes 68)."""
    lens = [0] * 60000
    for at, n in ((0, 100), (31, 3), (32, 64), (20000, 700), (20001, 1), (40000, 129), (59999, 300)):
        lens[at] = n
    op, q, k, v, d_o, cu = make(lens, 2, 1, 64, dtype, cuda_device, first=1, tail=7, seed=50)
    check(op, q, k, v, d_o, cu)
    o, lse = forward(op, q, k, v, cu)
    backward(op, q, k, v, o, lse, d_o, cu)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    start.record()
    op.pm_attention_packed_forward(q, k, v, cu, o, lse)
    end.record()
    end.synchronize()
    assert start.elapsed_time(end) < 20.0


@pytest.mark.parametrize("dtype", [BF, F])
def test_starts_that_do_not_ascend(cuda_device, dtype):
    """Whatever cu_seqlens holds, nothing outside the tensors is written, and the next call is right."""
    rng = random.Random(5)
    lens = [rng.randint(0, 9) for _ in range(700)]
    op, q, k, v, d_o, cu = make(lens, 2, 1, 64, dtype, cuda_device, seed=51)
    T = q.shape[0]
    bad = cu.clone()
    for i in range(0, 701, 3):
        bad[i] = rng.choice([rng.randint(-2 ** 31, 2 ** 31 - 1), rng.randint(-20, T + 20)])
    room = [torch.full((T + 64, 2, 64), 3.0, dtype=dtype, device=cuda_device) for _ in range(4)]
    stats = torch.full((2 * T + 64,), 3.0, device=cuda_device)
    o, dq, dk, dv = (r[32:32 + T, :n] for r, n in zip(room, (2, 2, 1, 1)))
    lse = stats[32:32 + 2 * T].view(2, T)
    op.pm_attention_packed_forward(q, k, v, bad, o, lse)
    op.pm_attention_packed_backward(q, k, v, o, lse, d_o, bad, dq, dk, dv)
    for r in room:
        assert (r[:32] == 3.0).all() and (r[32 + T:] == 3.0).all()
    assert (room[2][:, 1] == 3.0).all() and (room[3][:, 1] == 3.0).all()
    assert (stats[:32] == 3.0).all() and (stats[32 + 2 * T:] == 3.0).all()
    op.pm_attention_packed_status()
    o, lse = forward(op, q, k, v, cu)
    wo, wl, bo, bl = R.attention_forward(q, k, v, cu, op.scale, True, dtype)
    within(o, wo, bo, "o")
