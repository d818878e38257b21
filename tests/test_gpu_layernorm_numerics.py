"""Layer norm through its C entry with every output full of NaN beforehand, so that what is left unwritten fails, and with bounds that a NaN
fails; each gradient of weight and bias alone; many rows.

Bounds, with u = 2^-24 and U8 = 2^-8.  A row's sums run over at most 32 terms in a lane, 6 levels of a tree and 16 wavefronts: 54 u relative to
the sum of magnitudes, with the products' own roundings below 1e-5, and twice that where two such sums meet (the backward).  A column's sum of
rows runs over ceil(rows / (workgroups x rows a workgroup holds)) rows of a lane, the groups of a workgroup (32 at most), the partial sums
of 64 slices and 6 levels of a tree, one after the other: u times their number, and 4 u for the products."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from test_gpu_layernorm import SHAPES, U8, bf, dev, host, inputs

from paper_2603_22370_amd import binding as fb

U = 2.0 ** -24


def inside(got, want, tol, name):
    bad = ~(np.abs(got - want) <= tol + 1e-30)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist())


def full(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def at(t):
    return None if t is None else t.data_ptr()


def column_terms(T, D):
    """Terms of a column's sum that are added one after the other."""
    lanes = 8 if D <= 64 else 16 if D <= 128 else 32 if D <= 256 else 64
    held = 256 // lanes if D <= 512 else 1
    groups = fb.faar_workspace_bytes(fb.OP_LAYERNORM_BWD, D, 16, T) // (2 * D * 4)       # at least the workgroups
    rows = -(-T // (held * max(1, min(groups, -(-T // held)))))
    return rows + held + -(-groups // 64) + 6 + 4


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", SHAPES + [(16384, 512), (10007, 1024), (40000, 64)])
@pytest.mark.parametrize("xbf", [True, False])
def test_every_entry_is_written(T, D, xbf):
    L = fb.lib()
    rng, x, g, b = inputs(T, D, xbf)
    gd, bd, xd, stream = torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), dev(x, xbf), fb._stream()
    size = lambda t: np.abs(t).mean(axis=1, keepdims=True)
    h, mean, rstd = full(T, D, dtype=torch.bfloat16), full(T), full(T)
    assert L.faar_layernorm_fwd(xd.data_ptr(), fb._dt(xd), T, D, gd.data_ptr(), bd.data_ptr(), 1e-5, h.data_ptr(), mean.data_ptr(), rstd.data_ptr(), stream) == 0
    h_w, m_w, r_w = bo.layernorm(x, g, b, 1e-5)
    inside(host(mean), m_w, 1e-5 * size(x)[:, 0], "mean")
    inside(host(rstd), r_w, 1e-5 * r_w, "rstd")
    made = r_w[:, None] * (np.abs(x) + size(x)) * np.abs(g) + np.abs(b)
    inside(host(h), h_w, U8 * np.abs(h_w) + 1e-5 * made, "h")

    dh1, dh2, res = (bf(rng.standard_normal((T, D)) * 1e-2) for _ in range(3))
    d1, d2, rd = dev(dh1), dev(dh2), dev(res)
    m, r = host(mean), host(rstd)
    dx_w, dg_w, db_w = bo.layernorm_backward(dh1 + dh2, x, g, m, r)
    xh = r[:, None] * (np.abs(x) + np.abs(m)[:, None])
    dh = np.abs(dh1 + dh2)
    made = r[:, None] * (np.abs(g) * dh + size(g * dh) + xh * size(g * dh * xh)) + np.abs(res)
    terms = column_terms(T, D) * U
    ws_bytes = fb.faar_workspace_bytes(fb.OP_LAYERNORM_BWD, D, 16, T)
    for want_dg, want_db in ((True, True), (True, False), (False, True), (False, False)):
        dx, dg, db = full(T, D, dtype=torch.bfloat16), full(D) if want_dg else None, full(D) if want_db else None
        ws = full(ws_bytes // 4) if want_dg or want_db else None
        assert L.faar_layernorm_bwd(d1.data_ptr(), d2.data_ptr(), None, xd.data_ptr(), fb._dt(xd), T, D, gd.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                    rd.data_ptr(), dx.data_ptr(), at(dg), at(db), at(ws), ws_bytes, stream) == 0
        inside(host(dx), dx_w + res, U8 * np.abs(dx_w + res) + 2e-5 * made, "dx")
        if want_dg:
            inside(host(dg), dg_w, terms * (dh * xh).sum(axis=0), "dg")
        if want_db:
            inside(host(db), db_w, terms * dh.sum(axis=0), "db")


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 512, 2048, 12000])
def test_constant_rows_are_the_bias(D):
    L, T = fb.lib(), 9
    rng, x, g, b = inputs(T, D, False)
    x[:] = np.arange(T)[:, None] * 0.5 - 2.0               # exact in the sums: the mean is the value itself
    gd, bd, xd = torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), dev(x, False)
    h, mean, rstd = full(T, D, dtype=torch.bfloat16), full(T), full(T)
    assert L.faar_layernorm_fwd(xd.data_ptr(), fb._dt(xd), T, D, gd.data_ptr(), bd.data_ptr(), 1e-5, h.data_ptr(), mean.data_ptr(), rstd.data_ptr(), fb._stream()) == 0
    inside(host(mean), x[:, 0], 0.0, "mean")
    inside(host(rstd), np.full(T, 1e-5 ** -0.5), 1e-6 * 1e-5 ** -0.5, "rstd")
    inside(host(h), np.tile(bf(b), (T, 1)), 0.0, "h")
