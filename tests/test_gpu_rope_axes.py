"""GPU parity of the rotary embedding over several position axes against the oracle, and its refusals.

Tolerance: an output is a cos - b sin in float32, rounded to bf16 (half a step, 2^-8).  Sine and cosine are those of a fraction of a turn
good to half a step of float32 at 1/2, 2^-25 turns = 1.9e-7 radians, taken to 2 steps (2.4e-7), and three float32 roundings follow
(1.8e-7): together below 1e-6 of |a| + |b|.  The 64-bit product of position and frequency is off by at most 2 half-steps of 2^-53 of
its value: at 2^31 radians 4.8e-7 more."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from workloads import synth

import paper_2603_22370_amd as faar
from paper_2603_22370_amd import binding as fb

U8 = 2.0 ** -8


def bf(a):
    return synth.round_to_bf16(np.asarray(a, dtype=np.float32)).astype(np.float64)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def setup(T, n_axes, half, edge, seed):
    rng = np.random.default_rng([T, n_axes, half, seed])
    pos = rng.integers(-edge // 4, edge, (n_axes, T)).astype(np.int32)
    axis = rng.integers(0, n_axes, half)
    freq = [10000.0 ** (-i / half) for i in range(half)]
    return rng, pos, axis, freq


def check(got, x, pos, axis, freq, dh, pairs, inverse, extra=0.0):
    want = bo.rope_axes(x, pos, axis, freq, dh, pairs, inverse)
    half, T = len(freq), x.shape[0]
    xh = np.abs(x.reshape(T, -1, dh))
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    size = np.zeros_like(xh)
    size[..., a] = size[..., b] = xh[..., a] + xh[..., b]
    tol = U8 * np.abs(want) * (size.reshape(T, -1) > 0) + (1e-6 + extra) * size.reshape(T, -1)
    bad = np.abs(host(got) - want) > tol                   # entries that are not rotated have tolerance 0
    assert not bad.any(), int(bad.sum())


CASES = [(1, 1, 1, 16, 16, 1, 512), (5, 2, 1, 64, 64, 3, 512), (3, 4, 2, 80, 64, 2, 512), (2051, 3, 1, 128, 128, 3, 1 << 20),
         (130, 16, 16, 72, 32, 2, 1 << 16), (9, 1, 1, 256, 256, 4, 1 << 31), (2048, 2, 2, 24, 16, 1, 1 << 31)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,n_q,n_k,dh,rot,n_axes,edge", CASES)
@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_inverse_and_in_place(T, n_q, n_k, dh, rot, n_axes, edge, pairs):
    rng, pos, axis, freq = setup(T, n_axes, rot // 2, min(edge, (1 << 31) - 1), 1)
    q, k = bf(rng.standard_normal((T, n_q * dh)) * 3.0), bf(rng.standard_normal((T, n_k * dh)))
    qd, kd, pd = dev(q), dev(k), torch.from_numpy(pos).cuda()
    extra = 2.3e-16 * edge
    for inverse in (False, True):
        yq, yk = faar.faar_rope_axes(qd, kd, n_q, n_k, dh, pd, axis, freq, pairs=pairs, inverse=inverse)
        check(yq, q, pos, axis, freq, dh, pairs, inverse, extra)
        check(yk, k, pos, axis, freq, dh, pairs, inverse, extra)
        assert np.array_equal(host(qd), q)
        # alone, in place, and as slices of one buffer with other columns around them
        assert torch.equal(faar.faar_rope_axes(qd, None, n_q, 0, dh, pd, axis, freq, pairs=pairs, inverse=inverse)[0], yq)
        buf = torch.full((T, (n_q + n_k) * dh + 24), 9.0, dtype=torch.bfloat16, device="cuda")
        vq, vk = buf[:, 8:8 + n_q * dh], buf[:, 16 + n_q * dh:16 + (n_q + n_k) * dh]
        vq.copy_(qd)
        vk.copy_(kd)
        faar.faar_rope_axes(vq, vk, n_q, n_k, dh, pd, axis, freq, pairs=pairs, inverse=inverse, out=(vq, vk))
        assert torch.equal(vq, yq) and torch.equal(vk, yk)
        assert bool((buf[:, :8] == 9).all()) and bool((buf[:, 8 + n_q * dh:16 + n_q * dh] == 9).all()) and bool((buf[:, 16 + (n_q + n_k) * dh:] == 9).all())


@pytest.mark.gpu
def test_equal_positions_on_every_axis_are_the_one_axis_embedding():
    S, H, dh = 96, 2, 128
    rng, _, axis, freq = setup(S, 3, dh // 2, 512, 2)
    x = bf(rng.standard_normal((S, H * dh)))
    ang = np.arange(S)[:, None] * np.asarray(freq)[None, :]
    want = faar.faar_rope(dev(x), H, torch.from_numpy(np.cos(ang).astype(np.float32)).cuda(), torch.from_numpy(np.sin(ang).astype(np.float32)).cuda())
    pos = torch.arange(S, dtype=torch.int32, device="cuda").repeat(3, 1)
    got, _ = faar.faar_rope_axes(dev(x), None, H, 0, dh, pos, axis, freq)
    # both are within 1e-6 of |a| + |b| (the tables' entries within 2^-24) of the same value, before the same rounding
    a = np.abs(x.reshape(S, H, 2, dh // 2)).sum(axis=2)
    size = np.concatenate([a, a], axis=-1).reshape(S, -1)
    w = host(want)
    assert np.all(np.abs(host(got) - w) <= 2 * U8 * np.abs(w) + 2e-6 * size)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 2050])
def test_streams_and_graphs_of_positions_that_change(T):
    H, dh = 3, 64
    rng, pos, axis, freq = setup(T, 2, dh // 2, 4096, 4)
    q, pd = dev(rng.standard_normal((T, H * dh))), torch.from_numpy(pos).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = faar.faar_rope_axes(q, None, H, 0, dh, pd, axis, freq)
    side.synchronize()
    assert torch.equal(got, faar.faar_rope_axes(q, None, H, 0, dh, pd, axis, freq)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, _ = faar.faar_rope_axes(q, None, H, 0, dh, pd, axis, freq)
    for step in range(3):
        pd.add_(1)
        held.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, faar.faar_rope_axes(q, None, H, 0, dh, pd, axis, freq)[0])


def test_refusals():
    L = fb.lib()
    p, odd, nul = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), None
    ax, fr = (ctypes.c_uint8 * 32)(*[i % 2 for i in range(32)]), (ctypes.c_double * 32)(*[0.5 ** i for i in range(32)])
    def call(q=p, ldq=128, n_q=2, k=p, ldk=64, n_k=1, T=4, dh=64, rot=64, pos=p, n_axes=2, axis=ax, freq=fr, flags=0, yq=p, ldyq=128, yk=p, ldyk=64):
        return L.faar_rope_axes(q, ldq, n_q, k, ldk, n_k, T, dh, rot, pos, n_axes, axis, freq, flags, yq, ldyq, yk, ldyk, nul)
    assert call(q=nul) == -1 and call(yq=nul) == -1 and call(pos=nul) == -1 and call(axis=None) == -1 and call(freq=None) == -1
    assert call(k=nul) == -1 and call(yk=nul) == -1                    # k and yk come together
    assert call(T=0) == -2 and call(n_q=0) == -2 and call(n_k=0) == -2 and call(dh=60) == -2 and call(dh=264, ldq=528, ldk=264) == -2
    assert call(rot=0) == -2 and call(rot=24) == -2 and call(rot=80) == -2 and call(n_axes=0) == -2 and call(n_axes=257) == -2
    assert call(ldq=120) == -2 and call(ldq=132) == -2 and call(ldyk=56) == -2
    assert call(n_axes=1) == -6                                        # an axis that is not there
    assert call(freq=(ctypes.c_double * 32)(*([float("inf")] * 32))) == -6
    assert call(flags=4) == -6 and call(q=odd) == -6 and call(yk=odd) == -6 and call(pos=ctypes.c_void_p(0x1002)) == -6
    assert call(ldyq=136) == -6                                        # in place with another row stride
