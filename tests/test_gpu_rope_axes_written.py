"""The rotation over several position axes into outputs full of NaN, with bounds that a NaN fails (they are those of test_gpu_rope_axes)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from test_gpu_rope_axes import CASES, U8, bf, dev, host, setup

import paper_2603_22370_amd as faar


@pytest.mark.gpu
@pytest.mark.parametrize("T,n_q,n_k,dh,rot,n_axes,edge", CASES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_every_entry_is_written(T, n_q, n_k, dh, rot, n_axes, edge, pairs, inverse):
    rng, pos, axis, freq = setup(T, n_axes, rot // 2, min(edge, (1 << 31) - 1), 3)
    q, k, half = bf(rng.standard_normal((T, n_q * dh)) * 3.0), bf(rng.standard_normal((T, n_k * dh))), rot // 2
    # q's output in rows of its own, k's in the middle of wider ones
    yq = torch.full((T, n_q * dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide = torch.full((T, n_k * dh + 32), float("nan"), dtype=torch.bfloat16, device="cuda")
    yk = wide[:, 16:16 + n_k * dh]
    faar.faar_rope_axes(dev(q), dev(k), n_q, n_k, dh, torch.from_numpy(pos).cuda(), axis, freq, pairs=pairs, inverse=inverse, out=(yq, yk))
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, half), slice(half, rot))
    for got, x in ((yq, q), (yk, k)):
        want = bo.rope_axes(x, pos, axis, freq, dh, pairs, inverse)
        size, xh = np.zeros((T, x.shape[1] // dh, dh)), np.abs(x.reshape(T, -1, dh))
        size[..., a] = size[..., b] = xh[..., a] + xh[..., b]
        size = size.reshape(T, -1)
        bad = ~(np.abs(host(got) - want) <= U8 * np.abs(want) * (size > 0) + (1e-6 + 2.3e-16 * edge) * size)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())
    assert bool(torch.isnan(wide[:, :16]).all()) and bool(torch.isnan(wide[:, 16 + n_k * dh:]).all())
