"""Sizes that packed attention refuses before anything reaches a GPU: more blocks than one launch can have."""
import ctypes as C

import pytest

from paper_1910_05124_b200 import binding as B
from paper_1910_05124_b200 import build

P = 1 << 30           # addresses that are never followed


@pytest.mark.parametrize("dtype", [B.PM_BF16, B.PM_F32])
@pytest.mark.parametrize("n_seqs,n_heads,n_kv_heads", [(1 << 24, 128, 128), (1 << 24, 200, 8), (1 << 22, 512, 1), (40000, 65535, 1)])
def test_more_blocks_than_a_launch_has(n_seqs, n_heads, n_kv_heads, dtype):
    build.build()
    L = B.lib()
    d = B.pm_attention_desc(dtype, n_heads, n_kv_heads, 64, n_seqs, 1, 100, 0.125)
    far = 1 << 36
    v = [C.byref(B.pm_head_view(P + i * far, n_heads * 64, 64)) for i in range(8)]
    for st in (L.pm_attention_packed_forward(C.byref(d), *v[:3], P + 9 * far, v[3], P + 10 * far, None),
               L.pm_attention_packed_backward(C.byref(d), *v[:4], P + 10 * far, v[4], P + 9 * far, *v[5:], P + 11 * far, 1 << 40, None)):
        assert L.pm_status_string(st).decode() == "PM_ERR_SHAPE" and "sequences" in L.pm_last_error(None).decode()
