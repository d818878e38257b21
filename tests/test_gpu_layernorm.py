"""GPU parity of layer norm, forward and backward, against the float64 oracle, and its refusals.

Tolerances.  u = 2^-24 is half a step of float32; a bf16 output is off by half a step of its own, 2^-8 of its value.  A row's sums run
over at most 64 terms in a lane and 8 levels of a tree: 72 u, 4.3e-6, relative to the sum of magnitudes; with the products' own
roundings below 1e-5.  xh = (x - mean) r carries that of the mean, r mean|x| 1e-5, besides its own; what a value of the output is made
of is therefore good to 1e-5 of the magnitudes it is made of, twice that where two such sums meet (the backward).  A column's sum runs
over at most 64 rows of a lane, a workgroup's groups and 32 partial sums of 16 slices: fewer than 150 terms one after the other, 9e-6."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from workloads import synth

import paper_2603_22370_amd as faar
from paper_2603_22370_amd import binding as fb

U8 = 2.0 ** -8
SHAPES = [(1, 8), (1, 2048), (7, 40), (67, 64), (33, 136), (300, 256), (5, 520), (65, 1032), (130, 2048), (9, 2056), (3, 6152), (2, 16384),
          (2500, 96), (2100, 512), (300, 16384), (6200, 520), (700, 4104)]


def dev(a, bf16=True):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if bf16 else t


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def bf(a):
    return synth.round_to_bf16(np.asarray(a, dtype=np.float32)).astype(np.float64)


def inputs(T, D, xbf, offset=3.0):
    rng = np.random.default_rng([T, D, 7])
    x = rng.standard_normal((T, D)) * 2.0 + offset
    x[:, ::17] *= 20.0
    x = bf(x) if xbf else x.astype(np.float32).astype(np.float64)
    return rng, x, rng.uniform(0.5, 1.5, D).astype(np.float32), rng.standard_normal(D).astype(np.float32)


def inside(got, want, tol):
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), float((np.abs(got - want) / tol).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("xbf", [True, False])
def test_forward_and_backward(T, D, xbf):
    rng, x, g, b = inputs(T, D, xbf)
    gd_, bd_ = torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda()
    size = lambda t: np.abs(t).mean(axis=1, keepdims=True)
    for bias in (b, None):
        h, mean, rstd = faar.faar_layernorm_fwd(dev(x, xbf), gd_, None if bias is None else bd_, 1e-5)
        h_want, m_want, r_want = bo.layernorm(x, g, bias, 1e-5)
        inside(host(mean), m_want, 1e-5 * size(x)[:, 0] + 1e-30)
        # the mean's error moves the variance in second order, the sum of squares by 72 u
        inside(host(rstd), r_want, 1e-5 * r_want)
        made = r_want[:, None] * (np.abs(x) + size(x)) * np.abs(g) + (0.0 if bias is None else np.abs(bias))
        inside(host(h), h_want, U8 * np.abs(h_want) + 1e-5 * made)
    dh1, dh2, dh3, res = (bf(rng.standard_normal((T, D)) * 1e-2) for _ in range(4))
    m, r = host(mean), host(rstd)
    for two, three, with_res, cols in ((1, 1, 1, 1), (0, 0, 0, 0), (1, 0, 1, 1)):
        dh = dh1 + two * dh2 + three * dh3
        dx, dg, db = faar.faar_layernorm_bwd(dev(dh1), dev(x, xbf), gd_, mean, rstd, dh2=dev(dh2) if two else None,
                                             dh3=dev(dh3) if three else None, d_res=dev(res) if with_res else None, want_dg=bool(cols),
                                             want_db=bool(cols))
        want, dg_want, db_want = bo.layernorm_backward(dh, x, g, m, r)
        want = want + with_res * res
        xh = r[:, None] * (np.abs(x) + np.abs(m)[:, None])
        gd = np.abs(g * dh)
        made = r[:, None] * (gd + size(gd) + xh * size(gd * xh)) + with_res * np.abs(res)
        inside(host(dx), want, U8 * np.abs(want) + 2e-5 * made)
        if cols:
            inside(host(dg), dg_want, 1e-5 * (np.abs(dh) * xh).sum(axis=0) + 1e-30)
            inside(host(db), db_want, 1e-5 * np.abs(dh).sum(axis=0) + 1e-30)
        else:
            assert dg is None and db is None


@pytest.mark.gpu
def test_rows_far_from_zero_and_constant_rows():
    """The variance is taken about the mean: rows at 1000 +- 1 keep theirs; a constant row has xh = 0 and h = b."""
    T, D = 8, 512
    rng, x, g, b = inputs(T, D, False)
    x = (rng.standard_normal((T, D)) + 1000.0).astype(np.float32).astype(np.float64)
    x[3] = 7.0
    h, mean, rstd = faar.faar_layernorm_fwd(dev(x, False), torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), 1e-5)
    want, m_want, r_want = bo.layernorm(x, g, b, 1e-5)
    rest = np.arange(T) != 3
    # the mean is off by 72 u of 1000, 4.3e-3 at most of a deviation of 1
    inside(host(h)[rest], want[rest], U8 * np.abs(want[rest]) + 4.4e-3 * np.abs(g) * r_want[rest, None])
    inside(host(h)[3], bf(b), U8 * np.abs(b))
    inside(host(rstd)[rest], r_want[rest], 3e-5 * r_want[rest])


@pytest.mark.gpu
def test_gradients_against_differences():
    """What the kernels return as gradients is the slope of what the forward kernel computes: sum(d * h) along a few directions, with
    steps of a size at which the rounding of h (2^-8, averaged over T * D outputs) stays small beside the change."""
    T, D = 64, 256
    rng, x, g, b = inputs(T, D, False, offset=0.5)
    d = bf(rng.standard_normal((T, D)))
    gd, bd = torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda()
    _, mean, rstd = faar.faar_layernorm_fwd(dev(x, False), gd, bd, 1e-5)
    dx, dg, db = faar.faar_layernorm_bwd(dev(d), dev(x, False), gd, mean, rstd, want_dg=True, want_db=True)
    def value(x_, g_, b_):
        h, _, _ = faar.faar_layernorm_fwd(dev(x_, False), dev(g_, False), dev(b_, False), 1e-5)
        return float((host(h) * d).sum())
    for kind, grad in (("x", host(dx)), ("g", host(dg)), ("b", host(db))):
        e = np.sign(grad) * 0.05                           # along the gradient's signs: the change is 0.1 sum |grad|
        at = lambda s: value(x + s * e if kind == "x" else x, g + s * e if kind == "g" else g, b + s * e if kind == "b" else b)
        slope = at(1.0) - at(-1.0)
        want = 0.1 * np.abs(grad).sum()
        # h is rounded at 2 T D places by 2^-9 of |h| <= 5 rms and independent: sqrt(2 T D) 2^-9 * 2 |d|; x: third-order terms, 0.05^2
        noise = 4.0 * np.sqrt(2.0 * T * D) * 2.0 ** -9 * 2.0
        assert abs(slope - want) <= noise + 0.01 * want, (kind, slope, want)


@pytest.mark.gpu
def test_runs_agree_and_other_streams_and_graphs():
    T, D = 515, 1032
    rng, x, g, b = inputs(T, D, True)
    xd, gd, bd, dd = dev(x), torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), dev(rng.standard_normal((T, D)))
    ws = faar.layernorm_workspace(T, D)
    def both():
        h, mean, rstd = faar.faar_layernorm_fwd(xd, gd, bd, 1e-5)
        return (h, *faar.faar_layernorm_bwd(dd, xd, gd, mean, rstd, want_dg=True, want_db=True, ws=ws))
    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_refusals():
    L = fb.lib()
    import ctypes
    p, odd, nul = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), None
    f = L.faar_layernorm_fwd
    assert f(p, 1, 4, 64, nul, p, 1e-5, p, p, p, nul) == -1
    assert f(p, 1, 4, 64, p, p, 1e-5, p, nul, p, nul) == -1
    assert f(p, 5, 4, 64, p, p, 1e-5, p, p, p, nul) == -3
    assert f(p, 1, 0, 64, p, p, 1e-5, p, p, p, nul) == -2
    assert f(p, 1, 4, 60, p, p, 1e-5, p, p, p, nul) == -2
    assert f(p, 1, 4, 16392, p, p, 1e-5, p, p, p, nul) == -2
    assert f(p, 1, 4, 64, p, p, -1.0, p, p, p, nul) == -6
    assert f(p, 1, 4, 64, p, p, float("nan"), p, p, p, nul) == -6
    assert f(p, 1, 4, 64, p, odd, 1e-5, p, p, p, nul) == -6
    ws = fb.faar_workspace_bytes(fb.OP_LAYERNORM_BWD, 64, 16, 4)
    assert ws >= 2 * 64 * 4
    assert fb.faar_workspace_bytes(fb.OP_LAYERNORM_BWD, 64, 16, 0) == 0 and fb.faar_workspace_bytes(fb.OP_LAYERNORM_BWD, 60, 16, 4) == 0
    b = L.faar_layernorm_bwd
    assert b(nul, nul, nul, p, 1, 4, 64, p, p, p, nul, p, nul, nul, nul, 0, nul) == -1
    assert b(p, nul, nul, p, 1, 4, 64, p, p, p, nul, nul, nul, nul, nul, 0, nul) == -1
    assert b(p, nul, nul, p, 9, 4, 64, p, p, p, nul, p, nul, nul, nul, 0, nul) == -3
    assert b(p, nul, nul, p, 1, 4, 16392, p, p, p, nul, p, nul, nul, nul, 0, nul) == -2
    assert b(p, nul, odd, p, 1, 4, 64, p, p, p, nul, p, nul, nul, nul, 0, nul) == -6
    assert b(p, nul, nul, p, 1, 4, 64, p, p, p, nul, p, odd, nul, p, ws, nul) == -6
    assert b(p, nul, nul, p, 1, 4, 64, p, p, p, nul, p, p, nul, nul, 0, nul) == -4
    assert b(p, nul, nul, p, 1, 4, 64, p, p, p, nul, p, nul, p, p, ws - 1, nul) == -4
