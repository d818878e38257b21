"""The rotation over several position axes at more rows than one row of a grid has workgroups for."""
import numpy as np
import pytest
import torch

from test_gpu_rope_axes import check

import paper_2603_22370_amd as faar


@pytest.mark.gpu
def test_more_rows_than_a_launch_has_threads_for():
    """2^26 + 5 rows, four a workgroup of 256: 2^32 threads and more."""
    T, dh = (1 << 26) + 5, 16
    x = torch.randn(4096, dh, device="cuda").to(torch.bfloat16)
    q = torch.empty(T, dh, dtype=torch.bfloat16, device="cuda")
    for at in range(0, T, 4096):
        q[at:at + 4096] = x[:T - at]
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None]
    freq = [10.0 ** (-i / 2) for i in range(dh // 2)]
    y = torch.full_like(q, float("nan"))
    faar.faar_rope_axes(q, None, 1, 0, dh, pos, [0] * (dh // 2), freq, out=(y, None))
    assert not bool(torch.isnan(y).any())
    rows = np.r_[0:50, (1 << 25) - 20:(1 << 25) + 20, (1 << 26) - 20:T]
    at = torch.from_numpy(rows).cuda()
    check(y[at], q[at].float().cpu().numpy().astype(np.float64), rows[None].astype(np.int64), [0] * (dh // 2), freq, dh, False, False, 2.3e-16 * T)
