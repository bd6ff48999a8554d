"""The workspace of packed attention's backward pass: any address at a multiple of four, nothing in it before, nothing written beside it."""
import ctypes as C
import math

import pytest
import torch

from test_gpu_packed_attention import BF, F, backward, forward, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(BF, 64), (BF, 128), (BF, 33), (F, 64)])
def test_alignment_and_size(cuda_device, dtype, D):
    import paper_1910_05124_b200 as pm
    from paper_1910_05124_b200 import binding as B
    op, q, k, v, d_o, cu = make([301, 0, 70], 3, 1, D, dtype, cuda_device, first=2, tail=9, seed=31)
    o, lse = forward(op, q, k, v, cu)
    want = backward(op, q, k, v, o, lse, d_o, cu)
    desc = B.pm_attention_desc(B.PM_BF16 if dtype == BF else B.PM_F32, 3, 1, D, 3, 1, q.shape[0], op.scale)
    need = pm.lib().pm_attention_packed_workspace_bytes(C.byref(desc))
    assert need % 4 == 0
    for first in (0, 1, 2, 3, 5):
        room = torch.full((need // 4 + 12,), math.nan, device=cuda_device)
        out = [torch.zeros(x.shape, dtype=dtype, device=cuda_device) for x in (q, k, v)]
        view = [C.byref(B.pm_head_view(x.data_ptr(), x.stride(0), x.stride(1))) for x in (q, k, v, o, d_o, *out)]
        st = pm.lib().pm_attention_packed_backward(C.byref(desc), *view[:4], lse.data_ptr(), view[4], cu.data_ptr(), *view[5:],
                                                   room[first:].data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert st == 0, pm.lib().pm_last_error(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, want[n]) for a, n in zip(out, ("dq", "dk", "dv"))), first
        assert room[:first].isnan().all() and room[first + need // 4:].isnan().all()
