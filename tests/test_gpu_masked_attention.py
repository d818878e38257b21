"""GPU parity of attention under masks (forward, backward, single tokens over caches) against the float64 oracle, its plan and refusals.

Tolerances, element by element, from what the kernels round.  u = 2^-24 and U8 = 2^-8 are half a step of float32 and of bf16.  The
float32 score of a key is off by at most e = u (2 (dh + 8) Z + 16 S + 16) with Z = scale sum |q| |k| and S the largest score that counts (the
matrix cores' sum, the cap's exponential and reciprocal, the bias), so its probability by e of itself; P and ds are then rounded to
bf16, and so is every output:
    o:   U8 |o| + (U8 + 2 e) sum P |v|
    dv:  U8 |dv| + sum (U8 + 2 e) P |dO|,  over the query heads that share the key / value head
    ds = P (dP - delta) slack is good to (U8 + 4 e) |ds| and to what delta is off by, times P slack; dq and dk sum that over keys and
    queries, times scale |k| and scale |q|.  delta = sum dO o: without the low bytes of o off by sum |dO| tol(o).  With them o is
    sum w v / sum w with weights P (1 + eps), |eps| <= U8 + 2 e, off by sum P eps (v - o) up to second order, and stored to 2^-15: delta
    is off by 1.02 (U8 + 2 e) sum P |dP - delta| + 2^-15 sum |dO| |o| and float32 sums of dh products, 64 u sum |dO| sum P |v|.
Denominators and the sums over keys run in float32 over at most a few thousand terms of one sign in 16 or more partial sums: below
1e-5, in e."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from workloads import synth

import paper_2603_22370_amd as faar
from paper_2603_22370_amd import binding as fb

U8, U = 2.0 ** -8, 2.0 ** -24


def bf(a):
    return synth.round_to_bf16(np.asarray(a, dtype=np.float32)).astype(np.float64)


def dev(a, bf16=True):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if bf16 else t


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def ints(a):
    return torch.tensor(list(a), dtype=torch.int32, device="cuda")


def tolerances(q, k, v, seqs, n_q, n_kv, dh, scale, causal, window, cap, slopes, d_o=None, low=True):
    rep = n_q // n_kv
    tol = {"o": np.zeros_like(q), "lse": np.zeros((n_q, q.shape[0])), "dq": np.zeros_like(q), "dk": np.zeros_like(k), "dv": np.zeros_like(v)}
    want = bo.masked_attention(q, k, v, seqs, n_q, n_kv, dh, scale, causal, window, cap, slopes, d_o)
    for qs, ql, ks, kl, prefix in seqs:
        if ql == 0 or kl == 0:
            continue
        ok = bo.allowed_keys(ql, kl, causal, prefix, window)
        gap = np.abs(np.arange(ql)[:, None] + (kl - ql) - np.arange(kl)[None, :])
        for h in range(n_q):
            cq, ck = slice(h * dh, (h + 1) * dh), slice(h // rep * dh, (h // rep + 1) * dh)
            qh, kh, vh = q[qs:qs + ql, cq], k[ks:ks + kl, ck], v[ks:ks + kl, ck]
            z = qh @ kh.T * scale
            th = np.tanh(z / cap) if cap else np.zeros_like(z)
            s = (cap * th if cap else z) - (0.0 if slopes is None else float(slopes[h])) * gap
            lse = want[1][h, qs:qs + ql]
            with np.errstate(invalid="ignore"):
                P = np.where(ok, np.exp(np.where(ok, s, 0.0) - np.where(np.isfinite(lse), lse, 0.0)[:, None]), 0.0)
            counts = P > 1e-12
            Z = np.where(counts, scale * (np.abs(qh) @ np.abs(kh).T), 0.0).max(axis=1)
            S = np.where(counts, np.abs(s) + (cap if cap else 0.0), 0.0).max(axis=1)
            e = (U * (2 * (dh + 8) * Z + 16 * S + 16) + 1e-5)[:, None]
            tol["lse"][h, qs:qs + ql] = e[:, 0] + U * np.abs(np.where(np.isfinite(lse), lse, 0.0)) + 1e-6
            to = U8 * np.abs(want[0][qs:qs + ql, cq]) + (U8 + 2 * e) * (P @ np.abs(vh))
            tol["o"][qs:qs + ql, cq] = to
            if d_o is None:
                continue
            do = d_o[qs:qs + ql, cq]
            slack = 1.0 - th * th
            dp = do @ vh.T
            raw = P * np.abs(dp - (P * dp).sum(axis=1, keepdims=True))
            ds = raw * slack
            # dP - delta are float32 sums themselves: u dh of their magnitudes
            off = (np.abs(do) * to).sum(axis=1, keepdims=True) + U * 2 * dh * (np.abs(do) @ np.abs(vh).T)
            # slack = 4 r (1 - r) with r = 1 / (1 + E): E is off by 2 u of itself (a step of the exponential), the sum by u, the
            # reciprocal by 2 u, so r by 5 u and slack by 4 |1 - 2 r| 5 u + 2 u of its products <= 22 u, absolutely: where the cap
            # saturates, slack itself is smaller than that
            ds = (U8 + 4 * e) * ds + P * slack * off + (22 * U * raw if cap else 0.0)
            tol["dq"][qs:qs + ql, cq] += scale * (ds @ np.abs(kh))
            tol["dk"][ks:ks + kl, ck] += scale * (ds.T @ np.abs(qh))
            tol["dv"][ks:ks + kl, ck] += ((U8 + 2 * e) * P).T @ np.abs(do)
    if d_o is not None:
        for name, w in zip(("dq", "dk", "dv"), want[2:]):
            tol[name] += U8 * np.abs(w)
    return want, tol


def inside(got, want, tol, name):
    bad = ~(np.abs(got - want) <= tol + 1e-30)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.abs(got - want)[bad].max()))


class Case:
    def __init__(self, seqs, n_q, n_kv, dh, causal=True, window=0, cap=0.0, slopes=False, Tq=None, Tk=None, fused=False, gain=1.5, same=True, seed=0):
        self.seqs, self.n_q, self.n_kv, self.dh, self.causal, self.window, self.cap, self.same = seqs, n_q, n_kv, dh, causal, window, cap, same
        self.Tq = Tq or max(qs + ql for qs, ql, *_ in seqs)
        self.Tk = self.Tq if same else Tk or max(ks + kl for _, _, ks, kl, _ in seqs)
        self.fused, self.scale = fused, dh ** -0.5
        rng = np.random.default_rng([seed, n_q, dh, self.Tq])
        self.slopes = np.float32([2.0 ** (-4.0 * (j + 1) / n_q) for j in range(n_q)]) if slopes else None
        self.q, self.k, self.v, self.d_o = (bf(rng.standard_normal((T, h * dh)) * g) for T, h, g in
                                            ((self.Tq, n_q, gain), (self.Tk, n_kv, gain), (self.Tk, n_kv, 1.0), (self.Tq, n_q, 0.1)))
        self.q_rows, self.k_rows = np.zeros(self.Tq, bool), np.zeros(self.Tk, bool)
        for qs, ql, ks, kl, _ in seqs:
            self.q_rows[qs:qs + ql] = True
            self.k_rows[ks:ks + kl] = True

    def device(self):
        """Rows of no sequence hold NaN in every input."""
        parts = []
        for t, rows in ((self.q, self.q_rows), (self.k, self.k_rows), (self.v, self.k_rows), (self.d_o, self.q_rows)):
            x = dev(t)
            x[torch.from_numpy(~rows).cuda()] = float("nan")
            parts.append(x)
        if self.fused:
            widths = [t.shape[1] for t in parts[:3]]
            parts[:3] = torch.cat(parts[:3], dim=1).split(widths, dim=1)
        qs, ql, ks, kl, pre = (ints(t) for t in zip(*self.seqs))
        prefix = pre if any(s[4] for s in self.seqs) else None
        a = faar.attention_description(self.n_q, self.n_kv, self.dh, self.Tq, self.Tk, qs, ql, None if self.same else ks, None if self.same else kl,
                                       prefix=prefix, window=self.window, causal=self.causal, cap=self.cap,
                                       slopes=None if self.slopes is None else torch.from_numpy(self.slopes).cuda())
        return a, parts

    def oracle(self, grad=True, low=True):
        return tolerances(self.q, self.k, self.v, self.seqs, self.n_q, self.n_kv, self.dh, self.scale, self.causal, self.window, self.cap, self.slopes,
                          self.d_o if grad else None, low)


def packed(lens, prefix=0, gap=0):
    """Sequences one behind the other, `gap` rows of none between them."""
    out, at = [], gap
    for i, n in enumerate(lens):
        out.append((at, n, at, n, prefix if i % 2 == 0 else 0))
        at += n + gap
    return out


RAGGED = packed([1, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 200], gap=2)
# queries that are the last of longer caches, more queries than keys, no keys at all, no queries
MIXED = [(0, 5, 0, 70, 0), (5, 40, 70, 40, 0), (45, 30, 110, 3, 2), (75, 7, 113, 0, 0), (82, 0, 113, 9, 0), (82, 1, 122, 130, 0), (84, 129, 253, 300, 40)]

CASES = {
    "one_token": Case(packed([1]), 1, 1, 64),
    "ragged": Case(RAGGED, 2, 1, 64, Tq=920),
    "ragged_128_capped": Case(RAGGED, 4, 2, 128, cap=5.0, Tq=920),
    "ragged_bias": Case(RAGGED, 4, 4, 64, slopes=True),
    "ragged_prefix": Case(packed([1, 40, 130, 64, 200, 3], prefix=70), 2, 2, 128),
    "prefix_cap_bias_fused": Case(packed([33, 140, 90], prefix=50, gap=3), 6, 2, 64, cap=20.0, slopes=True, fused=True),
    "window": Case(packed([300, 65, 129]), 2, 1, 128, window=17),
    "window_of_one": Case(packed([70, 5]), 2, 2, 64, window=1),
    "window_64_bias": Case(packed([257, 100]), 3, 1, 64, window=64, slopes=True),
    "window_prefix": Case(packed([300, 200], prefix=100), 2, 2, 64, window=90, cap=50.0),
    "whole_sequences": Case(packed([1, 100, 64, 129, 300], gap=1), 2, 2, 80, causal=False, Tq=700),
    "whole_window_cap_bias": Case(packed([100, 270]), 4, 1, 128, causal=False, window=40, cap=10.0, slopes=True),
    "mixed_causal": Case(MIXED, 4, 2, 64, same=False, Tk=560, Tq=220),
    "mixed_whole_bias": Case(MIXED, 2, 1, 128, causal=False, slopes=True, same=False, Tk=560, Tq=220),
    "mixed_window_capped": Case(MIXED, 2, 2, 64, window=30, cap=3.0, same=False, Tk=560, Tq=220),
    "high_cap": Case(packed([150, 80]), 2, 1, 64, cap=100.0, gain=6.0),
    "sharp": Case(packed([200, 90]), 2, 2, 128, gain=8.0),
    "saturated_cap": Case(packed([200, 90]), 2, 2, 64, cap=4.0, gain=8.0),
    "heads_of_8": Case(packed([70, 33]), 4, 2, 8),
    "heads_of_24": Case(packed([70, 130]), 2, 1, 24, cap=8.0),
    "heads_of_96": Case(packed([70, 130, 64]), 2, 1, 96, cap=8.0),
    "heads_of_104": Case(packed([200, 33]), 2, 2, 104, causal=False, window=50),
    "heads_of_72": Case(packed([70, 130]), 2, 1, 72, slopes=True),
    "heads_of_120_fused": Case(packed([65, 130]), 3, 3, 120, fused=True),
    "one_key_value_head": Case(packed([129, 40]), 16, 1, 64, cap=30.0),
    # more work items than the device holds at once
    "many": Case(packed([130, 1, 200, 128, 65, 250] * 3, gap=1), 32, 8, 64, cap=5.0),
    "many_128": Case(packed([130, 1, 200, 128, 65, 250] * 2), 32, 4, 128, slopes=True),
    "many_whole_96": Case(packed([130, 33, 200, 129] * 3), 32, 32, 88, causal=False),
    "many_windows": Case(packed([300] * 5, prefix=40), 32, 2, 72, window=70, cap=90.0, slopes=True, fused=True),
    # few and many heads and keys beside one another: tiles in pieces, whole, and of many query heads
    "one_head_long": Case(packed([1300, 700]), 1, 1, 128, cap=20.0),
    "few_queries_long_keys": Case([(0, 3, 0, 1900, 0), (3, 40, 1900, 700, 0), (43, 0, 2600, 10, 0)], 4, 1, 64, same=False, slopes=True),
    "pairs_of_heads": Case(packed([130, 64, 200, 129, 65] * 3), 64, 32, 32, cap=5.0),
    "quads_of_heads": Case(packed([130, 64, 200, 129, 65] * 3), 64, 16, 24, window=100),
    "long": Case(packed([1500, 37]), 1, 1, 64, cap=30.0),
    # every sequence at the start of a place of 160 rows, and queries and keys in places of different sizes
    "padded": Case([(160 * b, n, 160 * b, n, 0) for b, n in enumerate([160, 1, 0, 97, 128])], 4, 2, 64, Tq=800, cap=50.0),
    "padded_apart": Case([(64 * b, n, 200 * b, m, 5) for b, (n, m) in enumerate([(64, 200), (1, 3), (10, 64), (0, 9)])], 2, 1, 96, same=False, Tq=256,
                         Tk=800),
}


def plan_layout(Tq, Tk, n, n_q, n_kv):
    """Where a plan has its lists: (places, bounds) of query items, key items, tiles of queries and of keys in pieces."""
    ceil = lambda x, y: -(-x // y)
    tq, tk = Tq // 128 + n, Tk // 64 + n
    eq = 0 if Tq // 128 * n_q >= 768 else min(ceil(512, n_q), tq * (ceil(ceil(Tk, 64), 8) - 1))
    ek = 0 if Tk // 64 * n_kv >= 1024 else min(ceil(1024, n_kv), tk * (ceil(n_q // n_kv * ceil(Tq, 64), 8) - 1))
    q_at, k_at = 16, 16 + 16 * (tq + eq)
    jq = k_at + 16 * (tk + ek)
    return (q_at, k_at, jq, jq + 8 * max(1, eq)), (tq + eq, tk + ek, eq, ek)


@pytest.mark.gpu
def test_plan_lists_every_tile_once():
    """Tiles cover the rows of every sequence once and lie inside it; their pieces cover the blocks that the masks leave once; what is in
    pieces has its own places; the most expensive come first."""
    in_pieces = set()
    for name, c in CASES.items():
        a, _ = c.device()
        plan = faar.faar_attention_plan(a).view(torch.int32).cpu().numpy()
        bad, no_bwd, nq, nk, jq, jk = plan[8:14]
        assert (bad, no_bwd) == (0, 0), name
        at, most = plan_layout(c.Tq, c.Tk, len(c.seqs), c.n_q, c.n_kv)
        assert nq <= most[0] and nk <= most[1] and jq <= most[2] and jk <= most[3], name
        for kind, (n_items, n_joins) in enumerate(((nq, jq), (nk, jk))):
            items = plan[at[kind]:at[kind] + 16 * n_items].reshape(-1, 16)
            joins = {int(w[0]): w for w in plan[at[2 + kind]:at[2 + kind] + 8 * n_joins].reshape(-1, 8)}
            assert len(joins) == n_joins
            tiles, used = {}, []
            for w in items:
                tiles.setdefault(int(w[0]), []).append(w)
            rows_seen = np.zeros(c.Tk if kind else c.Tq, int)
            for row0, pieces in tiles.items():
                pieces.sort(key=lambda w: w[7 if kind else 6])
                w = pieces[0]
                qs, ql, ks, kl, pre = next(s for s in c.seqs if s[2 * kind] <= row0 < s[2 * kind] + s[2 * kind + 1])
                start, length, size = (ks, kl, 64) if kind else (qs, ql, 128)
                rows = int(w[1])
                assert (row0 - start) % size == 0 and rows == min(size, start + length - row0), name
                rows_seen[row0:row0 + rows] += 1
                ok = bo.allowed_keys(ql, kl, c.causal, pre, c.window)
                if kind:
                    assert tuple(w[2:7]) == (row0 - ks, qs, ql, kl - ql, min(pre, kl)), name
                    i = np.flatnonzero(ok[:, row0 - ks:row0 - ks + rows].any(axis=1))
                    want = c.n_q // c.n_kv * (i[-1] // 64 + 1 - i[0] // 64) if i.size else 0
                    spans, slots = [(int(p[7]), int(p[8])) for p in pieces], [int(p[9]) for p in pieces]
                    assert spans[0][0] == 0 and spans[-1][1] == want, (name, spans, want)
                else:
                    assert tuple(w[2:6]) == (kl - ql + row0 - qs, ks, kl, min(pre, kl)), name
                    j = np.flatnonzero(ok[row0 - qs:row0 - qs + rows].any(axis=0))
                    spans, slots = [(int(p[6]), int(p[7])) for p in pieces], [int(p[8]) for p in pieces]
                    if j.size:
                        assert spans[0][0] == j[0] // 64 and spans[-1][1] == j[-1] // 64 + 1, (name, spans)
                assert all(x[1] == y[0] and x[0] < x[1] for x, y in zip(spans, spans[1:])), (name, spans)
                if len(pieces) == 1:
                    assert slots == [-1] and row0 not in joins
                else:
                    in_pieces.add(kind)
                    assert tuple(joins[row0][1:4]) == (rows, slots[0], len(pieces)) and slots == list(range(slots[0], slots[0] + len(pieces)))
                    used += slots
            assert np.array_equal(rows_seen, (c.k_rows if kind else c.q_rows).astype(int)), name
            assert sorted(used) == list(range(len(used))) and len(used) <= 2 * most[2 + kind], name
            costs = (items[:, 8] - items[:, 7]) if kind else (items[:, 7] - items[:, 6])
            assert len(costs) == 0 or (np.diff(costs) <= costs.max() // 64 + 1).all(), name
    assert in_pieces == {0, 1}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_forward_and_backward(name):
    c = CASES[name]
    (o_w, lse_w, dq_w, dk_w, dv_w), tol = c.oracle()
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    ws = faar.attention_masked_workspace(a, backward=True)
    out = torch.full((c.Tq, c.n_q * c.dh), 7.0, dtype=torch.bfloat16, device="cuda")
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v, out=out, ws=ws)
    rows, keys = c.q_rows, c.k_rows
    assert (host(o)[~rows] == 7.0).all()                   # rows of no sequence are left as they were
    inside(host(o)[rows], o_w[rows], tol["o"][rows], "o")
    got = host(stats.lse)[:, rows]
    none = np.isneginf(lse_w[:, rows])
    assert np.array_equal(np.isneginf(got), none)
    inside(got[~none], lse_w[:, rows][~none], tol["lse"][:, rows][~none], "lse")
    assert not host(o)[rows][none.any(axis=0)].any()       # a query that sees no key
    for low in (True, False):
        if not low:
            stats, (_, tol) = faar.AttentionStats(stats.lse, None), c.oracle(low=False)
        grads = [fb._zeros_like_rows(t).fill_(7.0) for t in (q, k, v)]
        grads = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats, out=grads, ws=ws)
        for g, w, r, n in zip(grads, (dq_w, dk_w, dv_w), (rows, keys, keys), ("dq", "dk", "dv")):
            assert (host(g)[~r] == 7.0).all(), n
            inside(host(g)[r], w[r], tol[n][r], n)



TOKENS = {  # lengths of the caches, capacity, n_q, n_kv, dh, window, cap, slopes
    "one": ([1], 64, 1, 1, 64, 0, 0.0, False),
    "ragged": ([0, 1, 31, 32, 33, 127, 128, 129, 700, 1000, 256], 1024, 4, 2, 128, 0, 0.0, False),
    "ragged_capped": ([0, 1, 31, 700, 129], 1000, 8, 1, 64, 0, 5.0, False),
    "bias": ([5, 300, 1100], 1100, 4, 4, 64, 0, 0.0, True),
    "cap_bias_window": ([5, 300, 1100, 64], 1100, 4, 2, 80, 200, 20.0, True),
    "window_of_one": ([5, 300], 320, 2, 1, 128, 1, 0.0, False),
    "many_heads_share": ([40, 333], 384, 80, 2, 64, 0, 0.0, False),
    "long_alone": ([9001], 9100, 2, 1, 128, 0, 30.0, False),
    "heads_of_96": ([40, 300, 128], 320, 4, 2, 96, 0, 10.0, False),
    "one_piece_each": ([170, 1, 0], 170, 8, 8, 64, 0, 0.0, True),
    "small_caches": ([40, 3, 17], 40, 4, 1, 24, 0, 0.0, False),
    "high_cap": ([300, 200], 300, 2, 2, 128, 0, 100.0, False),
}


def token_case(name):
    lens, cap_rows, n_q, n_kv, dh, window, cap, slopes = TOKENS[name]
    n = len(lens)
    rng = np.random.default_rng([n, dh, cap_rows])
    q, k, v = (bf(rng.standard_normal((T, h * dh)) * 1.5) for T, h in ((n, n_q), (n * cap_rows, n_kv), (n * cap_rows, n_kv)))
    seqs = [(b, 1, b * cap_rows, L, 0) for b, L in enumerate(lens)]
    sl = np.float32([2.0 ** (-4.0 * (j + 1) / n_q) for j in range(n_q)]) if slopes else None
    return lens, cap_rows, n_q, n_kv, dh, window, cap, sl, q, k, v, seqs


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(TOKENS))
def test_single_tokens(name):
    lens, cap_rows, n_q, n_kv, dh, window, cap, sl, q, k, v, seqs = token_case(name)
    n = len(lens)
    (o_w, lse_w), tol = tolerances(q, k, v, seqs, n_q, n_kv, dh, dh ** -0.5, True, window, cap, sl)
    kd, vd = dev(k), dev(v)
    for b, L in enumerate(lens):                           # what the caches hold behind their lengths does not matter
        kd[b * cap_rows + L:(b + 1) * cap_rows] = float("nan")
        vd[b * cap_rows + L:(b + 1) * cap_rows] = float("nan")
    a = faar.attention_description(n_q, n_kv, dh, n, n * cap_rows, ints(b * cap_rows for b in range(n)), ints(lens), single=True, window=window,
                                   cap=cap, slopes=None if sl is None else torch.from_numpy(sl).cuda())
    plan = faar.faar_attention_plan(a)
    words = plan.view(torch.int32).cpu().numpy()
    cols = n_kv * -(-(n_q // n_kv) // 32)
    target, pieces = 0 if n * cap_rows <= 512 else -(-512 // cols), int(words[10])
    assert pieces <= n + target
    items, first = words[16:16 + 16 * pieces].reshape(-1, 16), 0
    for b, L in enumerate(lens):                           # the pieces of a cache follow one another and end with it
        mine = items[items[:, 0] == b]
        assert len(mine) == mine[0, 4] and words[16 + 16 * (n + target) + 2 * b] == first
        at = b * cap_rows + (max(0, L - window) if window else 0)
        for _, row, keys, gap, *_ in mine:
            assert row == at and keys >= 0 and gap == L - 1 - (row - b * cap_rows)
            at += keys
        assert at == b * cap_rows + L
        first += len(mine)
    o, stats = faar.faar_attention_masked_fwd(a, plan, dev(q), kd, vd)
    inside(host(o), o_w, tol["o"], "o")
    none, lse = np.isneginf(lse_w), host(stats.lse)
    assert np.array_equal(np.isneginf(lse), none) and stats.o_low is None
    inside(lse[~none], lse_w[~none], tol["lse"][~none], "lse")
    again, none = faar.faar_attention_masked_fwd(a, plan, dev(q), kd, vd, want_lse=False)
    assert none is None and torch.equal(again, o)


@pytest.mark.gpu
def test_equal_causal_sequences_are_the_causal_attention():
    n_seq, S, n_q, n_kv, dh = 3, 160, 4, 2, 128
    c = Case(packed([S] * n_seq), n_q, n_kv, dh)
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    o, lse = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    o2, lse2 = faar.faar_attention_fwd(q, k, v, n_seq, n_q, n_kv)
    (_, _, *_), tol = c.oracle(low=False)
    inside(host(o), host(o2), 2 * tol["o"], "o")           # each within tol of the same value
    inside(host(lse.lse), host(lse2), 2 * tol["lse"], "lse")
    for x, y, n in zip(faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, lse), faar.faar_attention_bwd(d_o, q, k, v, o2, lse2, n_seq, n_q, n_kv),
                       ("dq", "dk", "dv")):
        inside(host(x), host(y), 2 * tol[n], n)


@pytest.mark.gpu
def test_gradients_against_differences():
    """What the backward returns is the slope of what the forward computes: sum(d_o * o) along the signs of each gradient.  The forward's
    result is a bf16 number at every place: its rounding errors (2^-9 of |o| at most, independent) stay below the noise stated."""
    c = Case(packed([90, 40], prefix=20), 2, 1, 64, cap=6.0, slopes=True, gain=1.0)
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    o, lse = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    grads = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, lse)
    value = lambda *t: float((host(faar.faar_attention_masked_fwd(a, plan, *t)[0]) * c.d_o).sum())
    for i, g in enumerate(grads):
        step = torch.sign(g.float()) * 2.0 ** -4
        ends = []
        for s in (1.0, -1.0):
            t = [q, k, v]
            t[i] = (t[i].float() + s * step).to(torch.bfloat16)
            ends.append((value(*t), t[i].float()))
        moved = ends[0][1] - ends[1][1]                    # what the rounding to bf16 left of the two steps
        want = float((moved * g.float()).sum())
        noise = 4.0 * np.sqrt(2.0 * o.numel()) * 2.0 ** -9 * float(o.float().abs().max()) * 0.1
        assert abs(ends[0][0] - ends[1][0] - want) <= noise + 0.03 * abs(want), (i, ends[0][0] - ends[1][0], want)


@pytest.mark.gpu
def test_runs_agree_and_rows_do_not_see_other_sequences():
    c = CASES["ragged_128_capped"]
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    def run(q, k, v, d_o):
        o, lse = faar.faar_attention_masked_fwd(a, plan, q, k, v)
        return (o, lse.lse, lse.o_low, *faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, lse))
    want = run(q, k, v, d_o)
    rows = torch.from_numpy(c.q_rows).cuda()
    part = lambda t: (t if t.shape[0] == c.Tq else t.t())[rows]
    for x, y in zip(run(q, k, v, d_o), want):
        assert torch.equal(part(x), part(y))
    # another last sequence changes nothing in the others, bit for bit
    last = c.seqs[-1][0]
    q2, k2, v2, d2 = (t.clone() for t in (q, k, v, d_o))
    for t in (q2, k2, v2, d2):
        t[last:] = 3.0
    got = run(q2, k2, v2, d2)
    rows[last:] = False
    for x, y in zip(got, want):
        assert torch.equal(part(x), part(y))


@pytest.mark.gpu
def test_graph_with_lengths_that_change_between_replays_and_other_streams():
    """Plan, forward and backward captured once; the lengths in their tensors are others at every replay."""
    n_q, n_kv, dh, Tq = 2, 1, 64, 400
    start, length = ints([0, 150]), ints([150, 200])
    a = faar.attention_description(n_q, n_kv, dh, Tq, Tq, start, length, cap=10.0)
    rng = np.random.default_rng(5)
    q, k, v, d_o = (dev(rng.standard_normal((Tq, h * dh))) for h in (n_q, n_kv, n_kv, n_q))
    plan, ws = faar.faar_attention_plan(a), faar.attention_masked_workspace(a, backward=True)
    def run():
        faar.faar_attention_plan(a, out=plan)
        o, lse = faar.faar_attention_masked_fwd(a, plan, q, k, v, ws=ws)
        return (o, *faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, lse, ws=ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = [t.clone() for t in run()]
    side.synchronize()
    for x, y in zip(run(), eager):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for lens in ([150, 200], [1, 250], [150, 0], [129, 64]):
        length.copy_(ints(lens))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for x, y in zip(got, run()):
            assert torch.equal(x, y), lens


@pytest.mark.gpu
def test_wrong_plans_and_lengths_are_answered_with_nan():
    c = CASES["ragged"]
    a, (q, k, v, d_o) = c.device()
    good = faar.faar_attention_plan(a)
    o, lse = faar.faar_attention_masked_fwd(a, good, q, k, v)
    all_nan = lambda *ts: all(bool(torch.isnan((t.lse if isinstance(t, faar.AttentionStats) else t).float()).all()) for t in ts)
    # a plan of another mask
    for change in (dict(window=9), dict(causal=False)):
        other = faar.attention_description(c.n_q, c.n_kv, c.dh, c.Tq, c.Tk, *(ints(t) for t in list(zip(*c.seqs))[:2]), **change)
        assert all_nan(*faar.faar_attention_masked_fwd(other, good, q, k, v))
        assert all_nan(*faar.faar_attention_masked_bwd(other, good, d_o, q, k, v, o, lse))
    # sequences outside the rows, of negative length, with a negative prefix, more query rows than there are
    for start, length, prefix in (([0, 900], [5, 21], None), ([-1, 30], [5, 21], None), ([0, 30], [-5, 21], None), ([0, 30], [2 ** 31 - 1, 1], None),
                                  ([0, 30], [5, 21], [0, -1]), ([0, 0], [500, 500], None)):
        b = faar.attention_description(c.n_q, c.n_kv, c.dh, c.Tq, c.Tk, ints(start), ints(length), prefix=None if prefix is None else ints(prefix))
        plan = faar.faar_attention_plan(b)
        assert all_nan(*faar.faar_attention_masked_fwd(b, plan, q, k, v)), (start, length)
        assert all_nan(*faar.faar_attention_masked_bwd(b, plan, d_o, q, k, v, o, lse)), (start, length)
    # caches of single tokens
    t = faar.attention_description(c.n_q, c.n_kv, c.dh, 2, c.Tk, ints([0, 900]), ints([5, 21]), single=True)
    assert all_nan(*faar.faar_attention_masked_fwd(t, faar.faar_attention_plan(t), q[:2], k, v))
    # keys that several sequences share: a forward, no backward
    s = faar.attention_description(c.n_q, c.n_kv, c.dh, 920, 920, ints([0, 100]), ints([100, 100]), ints([1, 1]), ints([600, 600]))
    k0, v0, q0 = (torch.nan_to_num(x) for x in (k, v, q))
    plan = faar.faar_attention_plan(s)
    o, lse = faar.faar_attention_masked_fwd(s, plan, q0, k0, v0)
    seqs = [(0, 100, 1, 600, 0), (100, 100, 1, 600, 0)]
    (o_w, _), tol = tolerances(host(q0), host(k0), host(v0), seqs, c.n_q, c.n_kv, c.dh, c.scale, True, 0, 0.0, None)
    inside(host(o)[:200], o_w[:200], tol["o"][:200], "o")
    assert all_nan(*faar.faar_attention_masked_bwd(s, plan, torch.nan_to_num(d_o), q0, k0, v0, o, lse))


@pytest.mark.gpu
def test_plan_of_very_many_tokens_over_one_cache():
    """A million tokens that see one cache of 2^30 rows: 2^43 blocks of keys in all, one piece each."""
    n, rows = 1 << 20, 1 << 30
    length = torch.full((n,), rows, dtype=torch.int32, device="cuda")
    length[5:7] = 0
    a = faar.attention_description(1, 1, 8, n, rows, torch.zeros_like(length), length, single=True)
    w = faar.faar_attention_plan(a).view(torch.int32)
    assert int(w[8]) == 0 and int(w[10]) == n
    items = w[16:16 + 16 * n].view(n, 16)
    assert torch.equal(items[:, 0], torch.arange(n, dtype=torch.int32, device="cuda")) and torch.equal(items[:, 2], length)
    assert not bool(items[:, 1].any()) and torch.equal(items[:, 3], length - 1) and bool((items[:, 4] == 1).all())


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets():
    """Keys and values whose rows lie 2^23 elements apart: the last ones are 5 billion elements in."""
    n, ld, dh = 600, 1 << 23, 64
    lens = [n]
    rng = np.random.default_rng(8)
    q, k, v = (bf(rng.standard_normal((T, dh))) for T in (1, n, n))
    big = torch.empty((n, ld), dtype=torch.bfloat16, device="cuda")
    kd, vd = big[:, 64:64 + dh], big[:, ld - dh:]
    kd.copy_(dev(k))
    vd.copy_(dev(v))
    (o_w, _), tol = tolerances(q, k, v, [(0, 1, 0, n, 0)], 1, 1, dh, dh ** -0.5, True, 0, 0.0, None)
    a = faar.attention_description(1, 1, dh, 1, n, ints([0]), ints(lens), single=True)
    inside(host(faar.faar_attention_masked_fwd(a, faar.faar_attention_plan(a), dev(q), kd, vd)[0]), o_w, tol["o"], "single")
    a = faar.attention_description(1, 1, dh, 1, n, ints([0]), ints([1]), ints([0]), ints(lens))
    inside(host(faar.faar_attention_masked_fwd(a, faar.faar_attention_plan(a), dev(q), kd, vd)[0]), o_w, tol["o"], "tiles")


@pytest.mark.gpu
def test_gradients_that_are_not_given_places():
    """Of q, k and v in one buffer they come in one buffer, else each in its own; rows of no sequence are 0."""
    for name in ("prefix_cap_bias_fused", "mixed_causal"):
        c = CASES[name]
        a, (q, k, v, d_o) = c.device()
        plan = faar.faar_attention_plan(a)
        o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
        given = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats, out=[fb._zeros_like_rows(t) for t in (q, k, v)])
        got = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats)
        assert all(torch.equal(x, y) for x, y in zip(got, given))
        assert not host(got[0])[~c.q_rows].any() and not host(got[2])[~c.k_rows].any()
        one = len({x.untyped_storage().data_ptr() for x in got}) == 1
        assert one == c.fused and [x.stride(0) for x in got] == [x.stride(0) for x in (q, k, v)]


@pytest.mark.gpu
def test_one_plan_for_layers_that_differ():
    """A plan depends on the sequences, the mask and the heads alone: layers with other widths, caps and biases read the same one."""
    seqs, plan = packed([33, 140, 90], prefix=50, gap=3), None
    for dh, cap, slopes in ((64, 20.0, True), (104, 0.0, False), (24, 100.0, False)):
        c = Case(seqs, 6, 2, dh, cap=cap, slopes=slopes)
        (o_w, _, dq_w, dk_w, dv_w), tol = c.oracle()
        a, (q, k, v, d_o) = c.device()
        plan = faar.faar_attention_plan(a) if plan is None else plan
        o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
        inside(host(o)[c.q_rows], o_w[c.q_rows], tol["o"][c.q_rows], "o")
        for g, w, n in zip(faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats), (dq_w, dk_w, dv_w), ("dq", "dk", "dv")):
            inside(host(g)[c.q_rows], w[c.q_rows], tol[n][c.q_rows], n)


@pytest.mark.gpu
def test_two_streams_at_once():
    """One plan, a workspace a stream: calls in flight together give what each gives alone."""
    c = CASES["one_head_long"]                             # tiles in pieces, which meet in the workspace
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    def run(q, ws):
        o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v, ws=ws)
        return (o, stats.lse, *faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats, ws=ws))
    inputs = [q, (-q).contiguous()]
    spaces = [faar.attention_masked_workspace(a, backward=True) for _ in inputs]
    want = [run(x, w) for x, w in zip(inputs, spaces)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in inputs], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = run(inputs[i], spaces[i])
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(t, u) for t, u in zip(x, y))


@pytest.mark.gpu
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (10.0, False), (100.0, False), (0.0, True)])
@pytest.mark.parametrize("n_q,n", [(1, 1300), (4, 150)])
def test_a_nan_that_is_seen_stays_one(n_q, n, cap, slopes):
    c = Case(packed([n, 70]), n_q, 1, 64, cap=cap, slopes=slopes)
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    row, head = n - 20, n_q - 1
    q[row, head * 64 + 5] = float("nan")
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    dq, _, _ = faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats)
    for t in (o, dq):
        bad = torch.isnan(t).view(-1, n_q, 64)
        assert bool(bad[row, head].all()) and int(bad.sum()) == 64
    assert bool(torch.isnan(stats.lse[head, row])) and int(torch.isnan(stats.lse).sum()) == 1
    # single tokens: in the first of two caches the key before the last
    t = faar.attention_description(n_q, 1, 64, 2, c.Tk, ints([0, n]), ints([n, 70]), single=True, cap=cap, slopes=None if not slopes else a._keep[-1])
    k[n - 2, 9] = float("nan")
    o, stats = faar.faar_attention_masked_fwd(t, faar.faar_attention_plan(t), q[:2].contiguous(), k, v)
    assert bool(torch.isnan(o[0]).all()) and not bool(torch.isnan(o[1]).any())
    assert bool(torch.isnan(stats.lse[:, 0]).all()) and not bool(torch.isnan(stats.lse[:, 1]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[700, 1, 3000], [100, 7, 0]])
def test_single_tokens_in_a_graph(lens):
    """Tokens generated one after the other by replays of one graph: the lengths grow by one, the plan follows."""
    n, cap_rows, n_q, n_kv, dh = len(lens), max(lens) + 8, 4, 2, 64
    rng = np.random.default_rng(11)
    q, k, v = (dev(rng.standard_normal((T, h * dh))) for T, h in ((n, n_q), (n * cap_rows, n_kv), (n * cap_rows, n_kv)))
    length = ints(lens)
    a = faar.attention_description(n_q, n_kv, dh, n, n * cap_rows, ints(b * cap_rows for b in range(n)), length, single=True, cap=30.0)
    plan, ws = faar.faar_attention_plan(a), faar.attention_masked_workspace(a)
    o = torch.empty_like(q)
    def token():
        faar.faar_attention_plan(a, out=plan)
        return faar.faar_attention_masked_fwd(a, plan, q, k, v, out=o, want_lse=False, ws=ws)[0]
    token()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        length.add_(1)
        token()
    for step in range(4):
        o.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        assert length.tolist() == [x + step + 1 for x in lens]
        assert torch.equal(got, token()) and not bool(torch.isnan(got).any())


def test_tensors_of_other_devices_are_refused(monkeypatch):
    class On:
        def __init__(self, device):
            self.get_device = lambda: device
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 77, raising=False)
    assert fb._raw_stream(On(1), None, On(1)) == 77
    for ts in ((On(0),), (On(1), On(0)), (On(1), None, On(-1))):
        with pytest.raises(ValueError, match="another device"):
            fb._raw_stream(*ts)


def test_refusals():
    L = fb.lib()
    p, odd, half, nul = 0x1000, 0x1004, 0x1002, None
    P = ctypes.c_void_p(p)
    def desc(**kw):
        a = fb.faar_attention()
        a.n_seq, a.Tq, a.Tk, a.q_start, a.q_len, a.n_q, a.n_kv, a.dh = 2, 64, 64, p, p, 4, 2, 64
        a.ldq = a.ldo = 256
        a.ldk = a.ldv = 128
        a.scale, a.cap, a.flags = 0.125, 0.0, 1
        for key, val in kw.items():
            setattr(a, key, val)
        return a
    bad = [(-1, dict(q_start=None)), (-1, dict(q_len=None)), (-1, dict(k_len=p)), (-1, dict(k_start=p)), (-1, dict(q_start=None, q_len=None)),
           (-2, dict(n_seq=0)), (-2, dict(n_seq=(1 << 20) + 1)), (-2, dict(Tq=0)), (-2, dict(Tq=(1 << 30) + 1)), (-2, dict(Tk=65)), (-2, dict(n_kv=3)),
           (-2, dict(n_q=0)), (-2, dict(n_q=4098)), (-2, dict(dh=60)), (-2, dict(dh=136)), (-2, dict(dh=0)),
           (-2, dict(q_start=None, q_len=None, k_start=p, k_len=p, Tq=3)), (-2, dict(Tq=1 << 30, Tk=1 << 30, n_q=4096, n_kv=1, ldq=4096 * 64, ldo=4096 * 64)),
           (-6, dict(window=-1)), (-6, dict(flags=2)), (-6, dict(scale=0.0)), (-6, dict(scale=float("nan"))), (-6, dict(scale=float("inf"))),
           (-6, dict(cap=-1.0)), (-6, dict(cap=float("inf"))), (-6, dict(cap=1e-45)), (-6, dict(q_start=half)), (-6, dict(prefix=half)), (-6, dict(slopes=half))]
    big = 1 << 40
    fwd = lambda a, plan=P, pb=big, q=P, k=P, v=P, o=P, lse=P, low=nul, ws=P, wb=big: \
        L.faar_attention_masked_fwd(a, plan, pb, q, k, v, o, lse, low, ws, wb, nul)
    bwd = lambda a, plan=P, pb=big, d_o=P, q=P, k=P, v=P, o=P, lse=P, low=nul, dq=P, dk=P, dv=P, ws=P, wb=big: \
        L.faar_attention_masked_bwd(a, plan, pb, d_o, q, k, v, o, lse, low, dq, dk, dv, ws, wb, nul)
    for code, kw in bad:
        a = desc(**kw)
        r = ctypes.byref(a)
        assert L.faar_attention_plan_bytes(r) == 0 and L.faar_attention_masked_workspace_bytes(r, 0) == 0, kw
        assert L.faar_attention_plan(r, P, big, nul) == code and fwd(r) == code and bwd(r) == code, kw
    for kw in (dict(ldq=248), dict(ldq=260), dict(ldk=120), dict(ldv=132), dict(ldo=0), dict(ldk=(1 << 24) + 8)):
        a = desc(**kw)
        r = ctypes.byref(a)
        assert fwd(r) == -2 and bwd(r) == -2 and L.faar_attention_plan_bytes(r) > 0, kw
    a = desc()
    r = ctypes.byref(a)
    pb, wf, wb = L.faar_attention_plan_bytes(r), L.faar_attention_masked_workspace_bytes(r, 0), L.faar_attention_masked_workspace_bytes(r, 1)
    assert pb >= 64 + 32 * (2 + 3) and wf > 0 and wb >= 4 * 64 * 4
    odd = ctypes.c_void_p(odd)
    assert L.faar_attention_plan(nul, P, pb, nul) == -1 and L.faar_attention_plan(r, nul, pb, nul) == -1
    assert L.faar_attention_plan(r, odd, pb, nul) == -6 and L.faar_attention_plan(r, P, pb - 1, nul) == -4
    for name in ("plan", "q", "k", "v", "o"):
        assert fwd(r, **{name: nul}) == -1 and fwd(r, **{name: odd}) == -6, name
    assert fwd(r, low=odd) == -6 and bwd(r, low=odd) == -6
    assert fwd(r, lse=ctypes.c_void_p(half)) == -6 and fwd(r, ws=nul) == -4 and fwd(r, wb=wf - 1) == -4 and fwd(r, pb=pb - 1) == -4
    for name in ("plan", "d_o", "q", "k", "v", "o", "dq", "dk", "dv"):
        assert bwd(r, **{name: nul}) == -1 and bwd(r, **{name: odd}) == -6, name
    assert bwd(r, lse=nul) == -1 and bwd(r, ws=nul) == -4 and bwd(r, wb=wb - 1) == -4 and bwd(r, pb=pb - 1) == -4
    t = desc(q_start=None, q_len=None, k_start=p, k_len=p, Tq=2)
    r = ctypes.byref(t)
    assert L.faar_attention_plan_bytes(r) > 0 and L.faar_attention_masked_workspace_bytes(r, 0) > 4 * 66 * 4
    assert L.faar_attention_masked_workspace_bytes(r, 1) == 0 and bwd(r) == -7 and fwd(r, low=P) == -7


def test_outputs_in_the_place_of_inputs_are_refused():
    L, nul, big = fb.lib(), None, 1 << 40
    a = fb.faar_attention()
    a.n_seq, a.Tq, a.Tk, a.q_start, a.q_len, a.n_q, a.n_kv, a.dh, a.scale = 1, 64, 64, 0x1000, 0x1000, 2, 2, 64, 0.125
    a.ldq = a.ldo = a.ldk = a.ldv = 128
    r, at = ctypes.byref(a), [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(10)]
    plan, ws, lse, d_o, q, k, v, o, dq, dk = at
    dv = ctypes.c_void_p(0x2000000)
    for out in (q, k, v):
        assert L.faar_attention_masked_fwd(r, plan, big, q, k, v, out, lse, nul, ws, big, nul) == -6
    for place in (d_o, q, k, v, o):
        for i in range(3):
            outs = [dq, dk, dv]
            outs[i] = place
            assert L.faar_attention_masked_bwd(r, plan, big, d_o, q, k, v, o, lse, nul, *outs, ws, big, nul) == -6
    a.scale = 2.0 ** 127
    assert L.faar_attention_plan(r, plan, big, nul) == -6
