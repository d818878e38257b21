"""CPU: the largest descriptions of attention under masks.  A launch has below 2^32 threads; what would need more is refused before anything
is launched."""
import ctypes

from paper_2603_22370_amd import binding as fb

P, BIG, NUL = ctypes.c_void_p(0x1000), 1 << 50, None


def description(**kw):
    a = fb.faar_attention()
    a.n_seq, a.Tq, a.Tk, a.q_start, a.q_len, a.n_q, a.n_kv, a.dh = 2, 64, 64, 0x1000, 0x1000, 4, 2, 8
    a.scale, a.flags = 0.125, 1
    for key, val in kw.items():
        setattr(a, key, val)
    a.ldq = a.ldo = a.n_q * a.dh
    a.ldk = a.ldv = a.n_kv * a.dh
    return a


def plan_bytes(a):
    return fb.lib().faar_attention_plan_bytes(ctypes.byref(a))


def workspace(a, backward):
    return fb.lib().faar_attention_masked_workspace_bytes(ctypes.byref(a), backward)


def test_grids_of_more_threads_than_a_launch_has():
    L = fb.lib()
    def refused(a):
        r = ctypes.byref(a)
        return plan_bytes(a) == 0 and workspace(a, 0) == 0 and L.faar_attention_plan(r, P, BIG, NUL) == -2 and \
            L.faar_attention_masked_fwd(r, P, BIG, P, P, P, P, P, NUL, P, BIG, NUL) == -2
    n = 1 << 20
    for heads, fits in ((8, True), (15, True), (16, False), (64, False)):
        a = description(n_seq=n, Tq=n, Tk=n, n_q=heads, n_kv=1)
        assert refused(a) != fits, heads
    # as many rows as there may be, forward alone; the backward has a workgroup for every 64 keys
    a = description(Tk=1 << 30, k_start=0x1000, k_len=0x1000, n_kv=1)
    r = ctypes.byref(a)
    assert plan_bytes(a) > 0 and workspace(a, 0) > 0 and workspace(a, 1) == 0
    assert L.faar_attention_masked_bwd(r, P, BIG, P, P, P, P, P, P, NUL, P, P, P, P, BIG, NUL) == -2
    a = description(Tk=1 << 29, k_start=0x1000, k_len=0x1000, n_kv=1)
    assert workspace(a, 1) > 0
    # single tokens: a workgroup of 256 for every piece and 32 query heads, and of 128 for every query head
    single = dict(q_start=None, q_len=None, k_start=0x1000, k_len=0x1000, n_seq=n, Tq=n, Tk=1 << 30)
    assert plan_bytes(description(n_q=16, n_kv=1, **single)) > 0 and plan_bytes(description(n_q=8, n_kv=8, **single)) > 0
    assert refused(description(n_q=32, n_kv=1, **single)) and refused(description(n_q=16, n_kv=16, **single))


def test_scales_whose_gradients_would_overflow():
    """Under a cap dq and dk are sums times 4 scale: at 2^126 that is infinite."""
    for scale, cap, fits in ((2.0 ** 126, 0.0, True), (2.0 ** 126, 50.0, False), (2.0 ** 125, 50.0, True), (2.0 ** 125, 1e30, True), (2.0 ** 126, 1e30, False)):
        a = description(scale=scale, cap=cap)
        assert (plan_bytes(a) > 0) == fits and (workspace(a, 1) > 0) == fits, (scale, cap)
        assert fits or fb.lib().faar_attention_plan(ctypes.byref(a), P, BIG, NUL) == -6


def test_gradients_in_one_place_are_refused():
    a = description(dh=64)
    at = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(12)]
    plan, d_o, q, k, v, o, lse, ws = at[:8]
    for dq, dk, dv in ((at[8], at[8], at[9]), (at[8], at[9], at[8]), (at[8], at[9], at[9])):
        assert fb.lib().faar_attention_masked_bwd(ctypes.byref(a), plan, BIG, d_o, q, k, v, o, lse, NUL, dq, dk, dv, ws, BIG, NUL) == -6
