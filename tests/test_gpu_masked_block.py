"""The operators of blocks that are not Llama3- or Qwen3-shaped, run together as a joint step runs them: the attention half of a block
with layer norm, rotary embedding over three axes and capped attention over packed documents, its four linears soft-quantised.

    h = layernorm(x);  q, k, v = linear(h);  q, k = rope_axes(q), rope_axes(k);  o = attention(q, k, v);  y = x + linear_o(o)
    loss = mse_scale ||y - y_fp||^2, back through all of it into the rounding variables of the four linears, into g, b and into x

Every operator is compared with the oracle on the inputs that it got here, within the bounds of its own tests (test_gpu_layernorm,
test_gpu_rope_axes, test_gpu_masked_attention), and the ends of the chain with the float64 chain.  On the way there are 14 tensors rounded
to bf16 (h, q, k, v, both rotated, o, the output, and their gradients back to dh); a rounding is off by at most half a step, 2^-8, of each
value and so at most 2^-8 / sqrt(3) of a tensor's norm where the places in the step are evenly spread; added up, 14 of them make 3.2e-2."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from oracle import faar_oracle as fo
from test_gpu_masked_attention import U8, bf, dev, host, inside, ints, packed, tolerances
from workloads import synth

import paper_2603_22370_amd as faar

pytestmark = pytest.mark.gpu

CHAIN = 14 * 2.0 ** -8 / np.sqrt(3.0)


def norm_error(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


class Half:
    """Sizes, inputs and the float64 chain."""
    def __init__(self):
        self.lens, self.n_q, self.n_kv, self.dh, self.D, self.rot = [70, 33, 130], 4, 2, 64, 256, 48
        self.cap, self.window, self.beta, self.lam, self.eps = 8.0, 90, 6.0, 0.01, 1e-5
        self.T, self.scale = sum(self.lens), self.dh ** -0.5
        rng = np.random.default_rng(17)
        T, D, dh = self.T, self.D, self.dh
        self.ms = 1.0 / (T * D)
        shapes = {"q": (self.n_q * dh, D), "k": (self.n_kv * dh, D), "v": (self.n_kv * dh, D), "o": (D, self.n_q * dh)}
        self.layers = {}
        for i, (n, (O, K)) in enumerate(shapes.items()):
            W = synth.student_t_weight(O, K, 900 + i, scale=0.05)
            q = fo.quant_rtn(W, True)
            self.layers[n] = (W, q["s_global"], q["scales"], synth.rounding_variables(O, K, 950 + i))
        self.x = bf(synth.activations(T, D, 23) + 0.3)
        self.g, self.b = rng.uniform(0.5, 1.5, D).astype(np.float32), (rng.standard_normal(D) * 0.2).astype(np.float32)
        self.y_fp = bf(self.x + rng.standard_normal((T, D)) * 0.2)
        self.pos = np.stack([np.arange(T) // 50, np.arange(T) % 50 // 7, np.arange(T) % 7]).astype(np.int32)
        self.axis, self.freq = [i % 3 for i in range(self.rot // 2)], [100.0 ** (-i / 24) for i in range(self.rot // 2)]
        self.seqs = packed(self.lens)

    def rope(self, x, inverse=False):
        return bo.rope_axes(x, self.pos, self.axis, self.freq, self.dh, inverse=inverse)

    def attention(self, q, k, v, d_o=None):
        return bo.masked_attention(q, k, v, self.seqs, self.n_q, self.n_kv, self.dh, self.scale, True, self.window, self.cap, None, d_o)

    def exact(self):
        Wq = {n: fo.soft_weight(*lay, self.beta) for n, lay in self.layers.items()}
        h, mean, r = bo.layernorm(self.x, self.g, self.b, self.eps)
        q, k, v = self.rope(h @ Wq["q"].T), self.rope(h @ Wq["k"].T), h @ Wq["v"].T
        o, _ = self.attention(q, k, v)
        y, L, dy = bo.block_output_loss(self.x, o @ Wq["o"].T, self.y_fp, self.ms)
        _, _, dq, dk, dv = self.attention(q, k, v, dy @ Wq["o"])
        dq, dk = self.rope(dq, inverse=True), self.rope(dk, inverse=True)
        dh = dq @ Wq["q"] + dk @ Wq["k"] + dv @ Wq["v"]
        dx, dg, db = bo.layernorm_backward(dh, self.x, self.g, mean, r)
        out = {"y": y, "L": L, "dx": dx + dy, "dg": dg, "db": db}
        for n, X, dY in (("q", h, dq), ("k", h, dk), ("v", h, dv), ("o", o, dy)):
            W, sg, sb, V = self.layers[n]
            out["dV_" + n] = fo.stage1_loss_and_grads(W, sg, sb, V, X, np.zeros((self.T, W.shape[0])), self.beta, self.lam, 0.0, dY_ext=dY)["dV"]
        return out


def test_joint_step_of_an_attention_half():
    c = Half()
    want = c.exact()
    T, D = c.T, c.D
    lin = {}
    for n, (W, _, _, V) in c.layers.items():
        Wd, Vd = dev(W), dev(V, False)
        sg, sc, _, _ = faar.faar_quant_rtn(Wd)
        lin[n] = dict(W=Wd, sg=sg, sc=sc, V=Vd, m=torch.zeros_like(Vd), u=torch.zeros_like(Vd),
                      losses=torch.zeros(3, dtype=torch.float32, device="cuda"))
    xd, gd, bd = dev(c.x), dev(c.g, False), dev(c.b, False)
    pos = torch.from_numpy(c.pos).cuda()
    start, length = ints([s[0] for s in c.seqs]), ints(c.lens)
    desc = faar.attention_description(c.n_q, c.n_kv, c.dh, T, T, start, length, window=c.window, cap=c.cap, scale=c.scale)
    plan, ws = faar.faar_attention_plan(desc), faar.attention_masked_workspace(desc, backward=True)

    # ---- forward
    forward = lambda n, X: faar.faar_linear_forward(lin[n]["W"], lin[n]["sg"], lin[n]["sc"], lin[n]["V"], c.beta, X)
    h, mean, rstd = faar.faar_layernorm_fwd(xd, gd, bd, c.eps)
    h_want, _, r_want = bo.layernorm(c.x, c.g, c.b, c.eps)
    size = lambda t: np.abs(t).mean(axis=1, keepdims=True)
    inside(host(h), h_want, U8 * np.abs(h_want) + 1e-5 * (r_want[:, None] * (np.abs(c.x) + size(c.x)) * np.abs(c.g) + np.abs(c.b)), "h")
    q0, k0, v = forward("q", h), forward("k", h), forward("v", h)
    q, k = faar.faar_rope_axes(q0, k0, c.n_q, c.n_kv, c.dh, pos, c.axis, c.freq)
    pair = lambda t: np.tile(np.abs(t).reshape(T, -1, c.dh).sum(axis=2, keepdims=True), (1, 1, c.dh)).reshape(T, -1)   # more than |a| + |b|
    for got, src, name in ((q, q0, "q"), (k, k0, "k")):
        w = c.rope(host(src))
        inside(host(got), w, U8 * np.abs(w) + 1e-6 * pair(host(src)), name)
    o, stats = faar.faar_attention_masked_fwd(desc, plan, q, k, v, ws=ws)
    d = forward("o", o)
    loss, dy, y = faar.faar_block_output_loss(xd, d, dev(c.y_fp), c.ms, want_y=True)

    # ---- backward
    def back(n, X, dY):
        lay = lin[n]
        O, K = lay["W"].shape
        Xt, _, ic = faar.faar_layer_prepare(lay["W"], lay["sg"], lay["sc"], X, None)
        dX = torch.empty((T, K), dtype=torch.bfloat16, device="cuda")
        faar.faar_layer_step(lay["W"], lay["sg"], lay["sc"], lay["V"], lay["m"], lay["u"], X, Xt, None, ic, c.beta, c.lam, 0.0, 1e-3, 0.9, 0.999,
                             1e-8, 1, lay["losses"], faar.layer_step_workspace(O, K, T, chained=True), dY_ext=dY, dX=dX, joint=True)
        return dX
    d_o = back("o", o, dy)
    dq, dk, dv = faar.faar_attention_masked_bwd(desc, plan, d_o, q, k, v, o, stats, ws=ws)
    (o_w, _, dq_w, dk_w, dv_w), tol = tolerances(host(q), host(k), host(v), c.seqs, c.n_q, c.n_kv, c.dh, c.scale, True, c.window, c.cap, None, host(d_o))
    for got, w, name in ((o, o_w, "o"), (dq, dq_w, "dq"), (dk, dk_w, "dk"), (dv, dv_w, "dv")):
        inside(host(got), w, tol[name], name)
    dq0, dk0 = faar.faar_rope_axes(dq, dk, c.n_q, c.n_kv, c.dh, pos, c.axis, c.freq, inverse=True)
    for got, src, name in ((dq0, dq, "dq0"), (dk0, dk, "dk0")):
        w = c.rope(host(src), inverse=True)
        inside(host(got), w, U8 * np.abs(w) + 1e-6 * pair(host(src)), name)
    dhs = [back(n, h, t) for n, t in (("q", dq0), ("k", dk0), ("v", dv))]
    dx, dg, db = faar.faar_layernorm_bwd(dhs[0], xd, gd, mean, rstd, dh2=dhs[1], dh3=dhs[2], d_res=dy, want_dg=True, want_db=True)
    dh, m, r = sum(host(t) for t in dhs), host(mean), host(rstd)
    dx_w, dg_w, db_w = bo.layernorm_backward(dh, c.x, c.g, m, r)
    xh, gdh = r[:, None] * (np.abs(c.x) + np.abs(m)[:, None]), np.abs(c.g * dh)
    made = r[:, None] * (gdh + size(gdh) + xh * size(gdh * xh)) + np.abs(host(dy))
    inside(host(dx), dx_w + host(dy), U8 * np.abs(dx_w + host(dy)) + 2e-5 * made, "dx")
    inside(host(dg), dg_w, 1e-5 * (np.abs(dh) * xh).sum(axis=0), "dg")
    inside(host(db), db_w, 1e-5 * np.abs(dh).sum(axis=0), "db")

    # ---- the ends against the exact chain
    assert norm_error(host(y), want["y"]) <= CHAIN and abs(loss.item() - want["L"]) <= 2 * CHAIN * want["L"]
    for got, name in ((dx, "dx"), (dg, "dg"), (db, "db")):
        e = norm_error(host(got), want[name])
        print(f"{name}: {e:.2e}", flush=True)
        assert e <= CHAIN, (name, e)
    for n in c.layers:                                     # zero initial state: m = (1 - beta1) dV
        e = norm_error(host(lin[n]["m"]) / 0.1, want["dV_" + n])
        print(f"dV[{n}]: {e:.2e}", flush=True)
        assert e <= CHAIN, (n, e)


def test_a_generated_token_continues_its_sequence():
    """The last token of each sequence, attended to as a single token over the cache of all keys, is the last row of the sequence's
    forward: same mask, same scores, same rotation at its position."""
    c = Half()
    T = c.T
    rng = np.random.default_rng(3)
    x, v = dev(rng.standard_normal((T, c.n_q * c.dh))), dev(rng.standard_normal((T, c.n_kv * c.dh)))
    y = dev(rng.standard_normal((T, c.n_kv * c.dh)))
    pos = torch.from_numpy(c.pos).cuda()
    q, k = faar.faar_rope_axes(x, y, c.n_q, c.n_kv, c.dh, pos, c.axis, c.freq)
    start, length = ints([s[0] for s in c.seqs]), ints(c.lens)
    kw = dict(window=c.window, cap=c.cap)
    a = faar.attention_description(c.n_q, c.n_kv, c.dh, T, T, start, length, **kw)
    whole, _ = faar.faar_attention_masked_fwd(a, faar.faar_attention_plan(a), q, k, v)
    last = torch.tensor([s[0] + s[1] - 1 for s in c.seqs], device="cuda")
    q1, _ = faar.faar_rope_axes(x[last].contiguous(), None, c.n_q, 0, c.dh, pos[:, last].contiguous(), c.axis, c.freq)
    assert torch.equal(q1, q[last])
    t = faar.attention_description(c.n_q, c.n_kv, c.dh, len(c.lens), T, start, length, single=True, **kw)
    one, _ = faar.faar_attention_masked_fwd(t, faar.faar_attention_plan(t), q1, k, v)
    _, tol = tolerances(host(q), host(k), host(v), c.seqs, c.n_q, c.n_kv, c.dh, c.scale, True, c.window, c.cap, None)
    inside(host(one), host(whole)[last.cpu().numpy()], 2 * tol["o"][last.cpu().numpy()], "o")
