"""Plans of attention under masks: sequences that share rows are found whatever the buffer's size and the sequences' order, and sequences
that share none are served in any order."""
import numpy as np
import pytest
import torch

from test_gpu_masked_attention import Case, inside, host, ints, packed, tolerances

import paper_2603_22370_amd as faar

BAD, NO_BACKWARD = 8, 9                # words of a plan's header


def verdicts(T, q, k=None, Tk=None):
    """(refused, no backward) of the plan of sequences given as (starts, lengths) of queries, and of keys."""
    a = faar.attention_description(2, 1, 64, T, Tk or T, *(ints(t) for t in q), *((None, None) if k is None else (ints(t) for t in k)))
    w = faar.faar_attention_plan(a).view(torch.int32)[:16].cpu()
    return int(w[BAD]), int(w[NO_BACKWARD])


@pytest.mark.gpu
@pytest.mark.parametrize("edge", [31, 32, 33, 63, 64, 100])
def test_shared_rows_are_found(edge):
    """Two sequences that meet at `edge`, that share one row there, or that leave one free, in order and the other way round, in a buffer
    with room to spare."""
    for first, second in (((0, edge), (edge, 70)), ((edge, 70), (0, edge))):
        for shift, shared in ((0, 0), (-1, 1), (1, 0)):
            a, b = ((s + (shift if s else 0), n) for s, n in (first, second))
            starts, lens = zip(a, b)
            assert verdicts(500, (starts, lens)) == (shared, shared)
            # keys alone: the forward may share them
            assert verdicts(500, ([0, 100], [10, 10]), (starts, lens), 600) == (0, shared)
    # one inside the other; the same rows twice; sequences of no rows share none, wherever they stand
    assert verdicts(500, ([0, 20], [100, 3])) == (1, 1)
    assert verdicts(500, ([20, 0], [3, 100])) == (1, 1)
    assert verdicts(500, ([7, 7], [1, 1])) == (1, 1)
    assert verdicts(500, ([400, 50, 0, 60], [100, 0, 100, 0])) == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 20, 5000])
def test_rows_of_many_sequences_in_any_order(n):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 90, n)
    gaps = rng.integers(0, 3, n)
    starts = np.cumsum(lens + gaps) - lens
    T = int(starts[-1] + lens[-1] + 700)
    order = rng.permutation(n)
    starts, lens = starts[order], lens[order]
    assert verdicts(T, (starts, lens)) == (0, 0)
    full = np.flatnonzero(lens)
    for i in rng.choice(full, 3):      # one row too many, behind or before: only where no gap is left
        for grow in ((0, 4), (-4, 4)):
            s, m = starts.copy(), lens.copy()
            s[i], m[i] = max(0, s[i] + grow[0]), m[i] + grow[1]
            used = np.zeros(T + 100, int)
            for a, b in zip(s, m):
                used[a:a + b] += 1
            want = int(used.max() > 1)
            assert verdicts(T, (s, m)) == (want, want), (i, grow)


@pytest.mark.gpu
def test_calls_with_shared_and_with_shuffled_rows():
    c = Case(packed([100, 90, 33, 0, 130], gap=2), 2, 1, 64)
    c.seqs = [c.seqs[i] for i in (3, 4, 0, 2, 1)]          # any order: the same results
    (o_w, lse_w, *want), tol = c.oracle()
    a, (q, k, v, d_o) = c.device()
    plan = faar.faar_attention_plan(a)
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    inside(host(o)[c.q_rows], o_w[c.q_rows], tol["o"][c.q_rows], "o")
    for g, w, n in zip(faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, stats), want, ("dq", "dk", "dv")):
        inside(host(g)[c.q_rows], w[c.q_rows], tol[n][c.q_rows], n)
    all_nan = lambda *ts: all(bool(torch.isnan(t.float()).all()) for t in ts)
    q, k, v, d_o = (torch.nan_to_num(t) for t in (q, k, v, d_o))
    # query rows of two sequences
    b = faar.attention_description(2, 1, 64, c.Tq, c.Tk, ints([0, 50]), ints([100, 60]))
    plan = faar.faar_attention_plan(b)
    o2, s2 = faar.faar_attention_masked_fwd(b, plan, q, k, v)
    assert all_nan(o2, s2.lse, *faar.faar_attention_masked_bwd(b, plan, d_o, q, k, v, o, stats))
    # key rows of two sequences, 300 of the buffer's more than 350 in all: a forward, no backward
    seqs = [(0, 100, 1, 170, 0), (100, 100, 51, 130, 0)]
    b = faar.attention_description(2, 1, 64, c.Tq, c.Tk, *(ints(t) for t in list(zip(*seqs))[:4]))
    assert 170 + 130 <= c.Tk
    plan = faar.faar_attention_plan(b)
    o3, s3 = faar.faar_attention_masked_fwd(b, plan, q, k, v)
    (o_w, _), tol = tolerances(host(q), host(k), host(v), seqs, 2, 1, 64, c.scale, True, 0, 0.0, None)
    inside(host(o3)[:200], o_w[:200], tol["o"][:200], "o")
    assert all_nan(*faar.faar_attention_masked_bwd(b, plan, d_o, q, k, v, o3, s3))
