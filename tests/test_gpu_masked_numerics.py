"""Attention under masks where its arithmetic is tried hardest, against the float64 oracle.

Bounds, element by element, with u = 2^-24 and U8 = 2^-8, half a step of float32 and of bf16.  The float32 score of a key is off by at most
e = u (2 (dh + 8) Z + 16 S + 16 + 8 A) + 1e-5, relative to its probability: Z = scale sum |q| |k| and S the largest |score| that counts
(the matrix cores' sum; the cap's series or its exponential and reciprocal, 16 half-steps of the score; the bias; the difference from the
maximum), 1e-5 the float32 sums over keys, and A the cap where cap log2(e) <= 1024, 3.4e-4 at most, and 0 where it is wider: a wide cap costs
a score nothing of its own precision.  P and ds are rounded to bf16, and so is every output:
    o:   U8 |o| + (U8 + 2 e) sum P |v|
    dv:  U8 |dv| + sum (U8 + 2 e) P |dO|
    dq, dk:  U8 |.| + scale sum |k| (or |q|) times the error of dz = P (dP - delta) slack, which is (U8 + 4 e) |dz|, 22 u P |dP - delta| of the slack
         (4 r (1 - r), r good to 5 u), P slack times what dP and delta are off by, and the product of the two errors: u 2 dh sum |dO| |v| and for delta
      without the low bytes of o   sum |dO| tol(o)
      with them                    1.02 (U8 + 2 e) sum P |dP - delta| + 2^-15 sum |dO| |o| + (64 + n / 16) u sum |dO| sum P |v|
    since then o = sum w v / sum w with w = P (1 + eps), |eps| <= U8 + 2 e, so that o is off by sum P eps (v - o) up to second order, by what
    it is stored to, 2^-15 of itself, and by float32 sums, of n keys in steps of 16.  The same holds for o and its low bytes taken together:
    o + low:  1.02 (U8 + 2 e) sum P |v - o| + 2^-15 |o| + (64 + n / 16) u sum P |v|

Norm-wise.  The error of a rounding to bf16 is at most U8 of the value and evenly spread, U8 / sqrt(3) = 2.26e-3 of it in the root mean square.
o and dv carry two that are independent (P's and their own), dq and dk three (dz's, that of P through delta, their own): 3.2e-3 and 3.9e-3 of
their norms.  Half as much again is allowed for: 4.8e-3 and 5.9e-3."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from test_gpu_masked_attention import CASES, Case, bf, dev, host, inside, ints, packed

import paper_2603_22370_amd as faar

U8, U = 2.0 ** -8, 2.0 ** -24


def bounds(q, k, v, seqs, n_q, n_kv, dh, scale, causal=True, window=0, cap=0.0, slopes=None, d_o=None, low=True, both=False):
    """(what the oracle gives, the bounds of o, lse, dq, dk, dv, and where `both` is wanted of o with its low bytes)"""
    rep, narrow = n_q // n_kv, cap if cap * 1.4426950408889634 <= 1024.0 else 0.0
    want = bo.masked_attention(q, k, v, seqs, n_q, n_kv, dh, scale, causal, window, cap, slopes, d_o)
    tol = {"o": np.zeros_like(q), "both": np.zeros_like(q), "lse": np.zeros((n_q, q.shape[0])), "dq": np.zeros_like(q), "dk": np.zeros_like(k),
           "dv": np.zeros_like(v)}
    for qs, ql, ks, kl, prefix in seqs:
        if ql == 0 or kl == 0:
            continue
        ok = bo.allowed_keys(ql, kl, causal, prefix, window)
        gap = np.abs(np.arange(ql)[:, None] + (kl - ql) - np.arange(kl)[None, :])
        for h in range(n_q):
            rows, keys = slice(qs, qs + ql), slice(ks, ks + kl)
            cq, ck = slice(h * dh, (h + 1) * dh), slice(h // rep * dh, (h // rep + 1) * dh)
            qh, kh, vh, oh = q[rows, cq], k[keys, ck], v[keys, ck], want[0][rows, cq]
            z = qh @ kh.T * scale
            th = np.tanh(z / cap) if cap else np.zeros_like(z)
            s = (cap * th if cap else z) - (0.0 if slopes is None else float(slopes[h])) * gap
            lse = np.where(np.isfinite(want[1][h, rows]), want[1][h, rows], 0.0)
            P = np.where(ok, np.exp(np.where(ok, s, -np.inf) - lse[:, None]), 0.0)
            counts = P > 1e-12
            Z = np.where(counts, scale * (np.abs(qh) @ np.abs(kh).T), 0.0).max(axis=1)
            S = np.where(counts, np.abs(s), 0.0).max(axis=1)
            e = (U * (2 * (dh + 8) * Z + 16 * S + 16 + 8 * narrow) + 1e-5)[:, None]
            eps = U8 + 2 * e
            sums = (64 + kl / 16) * U
            tol["lse"][h, rows] = e[:, 0] + U * np.abs(lse) + 1e-6
            tol["o"][rows, cq] = U8 * np.abs(oh) + eps * (P @ np.abs(vh))
            stored = 2.0 ** -15 * np.abs(oh) + sums * (P @ np.abs(vh))
            if both:
                spread = np.stack([(P * np.abs(vh[None, :, i] - oh[:, None, i])).sum(axis=1) for i in range(dh)], axis=1)
                tol["both"][rows, cq] = 1.02 * eps * spread + stored
            if d_o is None:
                continue
            do = d_o[rows, cq]
            slack, dp = 1.0 - th * th, do @ vh.T
            raw = P * np.abs(dp - (P * dp).sum(axis=1, keepdims=True))
            off = U * 2 * dh * (np.abs(do) @ np.abs(vh).T)
            if low:
                off = off + 1.02 * eps * raw.sum(axis=1, keepdims=True) + (np.abs(do) * stored).sum(axis=1, keepdims=True)
            else:
                off = off + (np.abs(do) * tol["o"][rows, cq]).sum(axis=1, keepdims=True)
            # with the slack off by t <= 22 u and dP - delta by d <= off: (x + d) (slack + t) - x slack = x t + slack d + t d
            dz = (U8 + 4 * e) * raw * slack + P * slack * off + (22 * U * (raw + P * off) if cap else 0.0)
            tol["dq"][rows, cq] += scale * (dz @ np.abs(kh))
            tol["dk"][keys, ck] += scale * (dz.T @ np.abs(qh))
            tol["dv"][keys, ck] += (eps * P).T @ np.abs(do)
    if d_o is not None:
        for name, w in zip(("dq", "dk", "dv"), want[2:]):
            tol[name] += U8 * np.abs(w)
    return want, tol


def bounds_of(c, low=True, both=False):
    return bounds(c.q, c.k, c.v, c.seqs, c.n_q, c.n_kv, c.dh, c.scale, c.causal, c.window, c.cap, c.slopes, c.d_o, low, both)


def forward_and_backward(c, want, tol):
    """-> (o, stats, (dq, dk, dv)) on the device, within the bounds."""
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    out = torch.full((c.Tq, c.n_q * c.dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v, out=out)
    rows, keys = c.q_rows, c.k_rows
    inside(host(o)[rows], want[0][rows], tol["o"][rows], "o")
    none = np.isneginf(want[1][:, rows])
    assert np.array_equal(np.isneginf(host(stats.lse)[:, rows]), none)
    inside(host(stats.lse)[:, rows][~none], want[1][:, rows][~none], tol["lse"][:, rows][~none], "lse")
    places = [torch.full_like(t, float("nan")) for t in (q, k, v)]
    if c.fused:
        places = [torch.full((c.Tq, q.stride(0)), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :t.shape[1]] for t in (q, k, v)]
    grads = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats, out=places)
    for g, w, r, n in zip(grads, want[2:], (rows, keys, keys), ("dq", "dk", "dv")):
        inside(host(g)[r], w[r], tol[n][r], n)
    return o, stats, grads


WIDE = {  # sequences, n_q, n_kv, dh, other arguments
    "heads_of_64": (packed([200, 33, 90], gap=1), 4, 2, 64, {}),
    "heads_of_80_bias_window": (packed([270, 70]), 2, 2, 80, dict(slopes=True, window=100)),
    "heads_of_128_prefix_bias": (packed([150, 129], prefix=40), 2, 1, 128, dict(slopes=True)),
    "whole_sequences_of_128": (packed([65, 200]), 2, 2, 128, dict(causal=False)),
    "in_pieces": (packed([1300, 40]), 1, 1, 64, {}),
}


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [60.0, 709.0, 710.0, 1e5, 1e7, 1e9, 1e30])
@pytest.mark.parametrize("name", list(WIDE))
def test_wide_caps(name, cap):
    """A cap far above the scores changes nothing, one of their size bends them, and none costs them precision."""
    seqs, n_q, n_kv, dh, more = WIDE[name]
    c = Case(seqs, n_q, n_kv, dh, cap=cap, gain=14.0 if cap == 710.0 else 6.0 if cap == 60.0 else 3.5, **more)     # scores of deviation 196, 36, 12
    forward_and_backward(c, *bounds_of(c))


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [60.0, 710.0, 1e4, 1e7, 1e30])
@pytest.mark.parametrize("dh,slopes", [(64, False), (80, True), (128, False)])
def test_wide_caps_of_single_tokens(cap, dh, slopes):
    lens, rows, n_q, n_kv = [700, 1, 130], 720, 4, 2
    rng = np.random.default_rng([dh, 3])
    q, k, v = (bf(rng.standard_normal((T, h * dh)) * 3.5) for T, h in ((3, n_q), (3 * rows, n_kv), (3 * rows, n_kv)))
    sl = np.float32([2.0 ** (-4.0 * (j + 1) / n_q) for j in range(n_q)]) if slopes else None
    want, tol = bounds(q, k, v, [(b, 1, b * rows, n, 0) for b, n in enumerate(lens)], n_q, n_kv, dh, dh ** -0.5, cap=cap, slopes=sl)
    a = faar.attention_description(n_q, n_kv, dh, 3, 3 * rows, ints(b * rows for b in range(3)), ints(lens), single=True, cap=cap,
                                   slopes=None if sl is None else torch.from_numpy(sl).cuda())
    o, stats = faar.faar_attention_masked_fwd(a, faar.faar_attention_plan(a), dev(q), dev(k), dev(v))
    inside(host(o), want[0], tol["o"], "o")
    inside(host(stats.lse), want[1], tol["lse"], "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_gradients_that_read_the_low_bytes_of_o(name):
    """Within the closer bounds that o to 16 bits gives delta; and o with its low bytes is o to 16 bits, but for what P's rounding costs."""
    c = CASES[name]
    want, tol = bounds_of(c, both=c.Tq <= 1000)
    o, stats, _ = forward_and_backward(c, want, tol)
    if c.Tq > 1000:
        return
    top = o.view(torch.int16).to(torch.int32) << 16
    whole = (top + (stats.o_low.to(torch.int32) << 8)).view(torch.float32)
    inside(host(whole)[c.q_rows], want[0][c.q_rows], tol["both"][c.q_rows], "o and its low bytes")


def off(got, want, rows):
    return float(np.linalg.norm(host(got)[rows] - want[rows]) / np.linalg.norm(want[rows]))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["sharp", "high_cap", "images"])
def test_norms_of_errors(name):
    """Where a softmax is sharp dP - delta is a small difference of large numbers: without the low bytes of o it carries their rounding."""
    c = CASES[name] if name in CASES else Case(packed([700, 300]), 2, 2, 80, causal=False, gain=3.0)
    (o_w, _, *want), _ = bounds_of(c)
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    grads = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats)
    without = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, faar.AttentionStats(stats.lse, None))
    errors = [off(g, w, r) for g, w, r in zip(grads, want, (c.q_rows, c.k_rows, c.k_rows))]
    plain = [off(g, w, r) for g, w, r in zip(without, want, (c.q_rows, c.k_rows, c.k_rows))]
    print(name, "o", off(o, o_w, c.q_rows), "dq dk dv", errors, "without", plain)
    assert off(o, o_w, c.q_rows) <= 4.8e-3 and errors[2] <= 4.8e-3
    assert errors[0] <= 5.9e-3 and errors[1] <= 5.9e-3
    assert torch.equal(grads[2], without[2])
    if name == "sharp":
        assert errors[0] <= 0.8 * plain[0] and errors[1] <= 0.8 * plain[1]


@pytest.mark.gpu
@pytest.mark.parametrize("name,seqs,n_q,n_kv,dh,more", [
    ("documents", packed([4500, 700, 1200]), 2, 1, 128, dict(cap=50.0)),
    ("window_bias", packed([7001]), 1, 1, 64, dict(window=1024, slopes=True)),
    ("whole", packed([2500, 1007], gap=5), 2, 2, 80, dict(causal=False)),
    ("continued", [(0, 130, 0, 5000, 0), (130, 3000, 5000, 3100, 0)], 2, 1, 64, dict(same=False))])
def test_long_sequences(name, seqs, n_q, n_kv, dh, more):
    c = Case(seqs, n_q, n_kv, dh, **more)
    forward_and_backward(c, *bounds_of(c))


def saturated(seqs, n_q, n_kv, dh, cap, **more):
    """Scores of +-cap: rows of q whose scores are all -cap and rows whose are all +cap in turn, every seventh with scores in between.  Columns of
    v from 2^-18 up to 2^9."""
    c = Case(seqs, n_q, n_kv, dh, cap=cap, **more)
    rng = np.random.default_rng([int(cap), dh])
    way = bf(rng.standard_normal(dh))
    size = 16.0 * cap / (c.scale * float((way * way).sum()))             # |z / cap| is 12 and more: tanh is 1 to 1e-10
    sign = np.where(np.arange(c.Tq) % 2 == 0, -1.0, 1.0)
    sign[np.arange(c.Tq) % 7 == 3] = 0.0
    c.q = np.tile(bf(size * sign[:, None] * way[None, :]), (1, n_q))
    loose = sign == 0.0
    c.q[loose] = bf(rng.standard_normal((int(loose.sum()), n_q * dh)) * 4.0)
    c.k = np.tile(bf(way[None, :] * rng.uniform(0.75, 1.25, (c.Tk, 1))), (1, n_kv))
    c.v = bf(c.v * np.tile(2.0 ** (np.arange(dh) * 28 // dh - 18.0), n_kv)[None, :])
    return c


ENDS = {"packed": (packed([130, 64, 1, 200], gap=1), 2, 2, 64, {}), "whole_128": (packed([90, 129]), 2, 1, 128, dict(causal=False)),
        "heads_of_80": (packed([150]), 1, 1, 80, {}), "in_pieces": (packed([1300, 33]), 1, 1, 64, {})}


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [50.0, 51.9, 52.1, 30.0])
@pytest.mark.parametrize("name", list(ENDS))
def test_scores_at_both_ends_of_their_cap(name, cap):
    """Up to a cap of 52 exponents have a fixed reference: a row whose scores are all -cap sums terms of 2^-110, and of +cap of 2^40."""
    seqs, n_q, n_kv, dh, more = ENDS[name]
    c = saturated(seqs, n_q, n_kv, dh, cap, **more)
    want, tol = bounds_of(c, both=c.Tq < 1000)
    o, stats, _ = forward_and_backward(c, want, tol)
    if c.Tq < 1000:
        top = o.view(torch.int16).to(torch.int32) << 16
        whole = (top + (stats.o_low.to(torch.int32) << 8)).view(torch.float32)
        inside(host(whole)[c.q_rows], want[0][c.q_rows], tol["both"][c.q_rows], "o and its low bytes")


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [50.0, 51.9])
@pytest.mark.parametrize("dh", [64, 128])
def test_single_tokens_at_both_ends_of_their_cap(cap, dh):
    rows, lens, n_q = 900, [800, 3, 130, 700], 2
    c = saturated([(b, 1, b * rows, n, 0) for b, n in enumerate(lens)], n_q, 1, dh, cap, same=False, Tk=4 * rows)
    want, tol = bounds(c.q, c.k, c.v, c.seqs, n_q, 1, dh, c.scale, cap=cap)
    a = faar.attention_description(n_q, 1, dh, 4, 4 * rows, ints(b * rows for b in range(4)), ints(lens), single=True, cap=cap)
    o, stats = faar.faar_attention_masked_fwd(a, faar.faar_attention_plan(a), dev(c.q), dev(c.k), dev(c.v))
    inside(host(o), want[0], tol["o"], "o")
    inside(host(stats.lse), want[1], tol["lse"], "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("dh", [64, 128])
def test_a_nan_stays_one_under_a_wide_cap(dh):
    c = Case(packed([150, 70]), 2, 1, dh, cap=1e4)
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    q[100, dh + 5] = float("nan")
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    dq, _, _ = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats)
    for t in (o, dq):
        bad = torch.isnan(t).view(-1, 2, dh)
        assert bool(bad[100, 1].all()) and int(bad.sum()) == dh
    assert bool(torch.isnan(stats.lse[1, 100])) and int(torch.isnan(stats.lse).sum()) == 1
