"""The operators of blocks that are not built like the Llama3- and Qwen3-shaped ones, as a user of this library runs them.

Between the quantised linears of such a block stand layer norm instead of RMSNorm, rotary embedding over several position axes
(time, height and width of image and video patches), and attention whose scores are capped by a tanh or carry a bias that falls
with the distance, over documents packed into one row of tokens, with prefixes, windows, or images that see themselves whole;
and, where the calibrated model answers, one token a sequence over a cache of keys and values.  `listed()` names cases of each,
`draw(rng)` gives further ones of the same ranges, `prepare` makes what a program holds before the call, `run` makes one pass
(the operators' plain form, or with `own` set the library's), `work` counts the bytes and operations no implementation avoids,
and `exact` computes the outputs in 64 bits from the operators' definitions.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
THETA = 10000.0


# ---- the cases --------------------------------------------------------------------------------------------------------
def listed() -> list[dict]:
    return [
        # joint calibration on one packed row: 24 documents of ragged lengths in 8192 tokens, capped scores, heads as in the
        # Qwen3-1.7B-shaped block; forward and backward
        _attention("train_packed_capped", 24, 8192, 16, 8, 128, cap=50.0, grad=True, cut=3),
        # the same with a distance bias and a window on long sequences, heads of 64, q, k and v in one fused buffer
        _attention("train_bias_window", 3, 7001, 16, 4, 64, slopes=True, window=1024, grad=True, fused=True, cut=5),
        # image encoder blocks: patches of 13 images in one row, every patch sees its whole image, heads of 80, no shared heads
        _attention("train_images", 13, 10007, 16, 16, 80, causal=False, grad=True, cut=7),
        # a long prompt behind a prefix that is seen from everywhere; forward alone, the largest case
        _attention("prompt_prefix_long", 1, 16384, 16, 8, 128, prefix=2048, cap=30.0, cut=0),
        # answering, one request: one token over 700 keys, where latency counts
        _token("token_one_request", 1, 1024, 8, 8, 64, cut=11),
        # answering, a batch: 96 requests with ragged caches of up to 8192 keys, capped scores
        _token("token_batch", 96, 8192, 16, 8, 128, cap=50.0, cut=13),
        # rotation of q and k of a video's patches, three axes, heads as in the Qwen3-1.7B-shaped block
        _rope("rope_video", 16384, 16, 8, 128, 128, 3),
        # its backward pass on image patches: two axes, pairs of neighbours, heads of 80 of which 64 are rotated, an odd row count
        _rope("rope_images_backward", 4999, 16, 16, 80, 64, 2, pairs=True, inverse=True),
        # the rotation of a batch of single tokens at far positions
        _rope("rope_tokens", 24, 16, 8, 128, 128, 3, far=True),
        # layer norm before the MLP half of a joint step, forward and backward with two consumers, the residual's gradient
        # and the gradients of weight and bias
        _norm("norm_train", 16384, 2048, grad=True),
        # a wide one on a float32 residual stream at an odd token count
        _norm("norm_wide_f32", 2999, 5120, x="f32", grad=True),
        # a few tokens' layer norm while answering
        _norm("norm_tokens", 24, 2048),
    ]


def _attention(name, n_seq, tokens, n_q, n_kv, dh, causal=True, prefix=0, window=0, cap=0.0, slopes=False, grad=False, fused=False, cut=0):
    return {"name": name, "kind": "attention", "n_seq": n_seq, "tokens": tokens, "n_q": n_q, "n_kv": n_kv, "dh": dh, "causal": causal,
            "prefix": prefix, "window": window, "cap": cap, "slopes": slopes, "grad": grad, "fused": fused, "cut": cut}


def _token(name, n_seq, cache, n_q, n_kv, dh, window=0, cap=0.0, slopes=False, cut=0):
    return {"name": name, "kind": "token", "n_seq": n_seq, "cache": cache, "n_q": n_q, "n_kv": n_kv, "dh": dh, "window": window, "cap": cap,
            "slopes": slopes, "cut": cut}


def _rope(name, T, n_q, n_k, dh, rot, axes, pairs=False, inverse=False, far=False):
    return {"name": name, "kind": "rope", "T": T, "n_q": n_q, "n_k": n_k, "dh": dh, "rot": rot, "axes": axes, "pairs": pairs,
            "inverse": inverse, "far": far}


def _norm(name, T, D, x="bf16", grad=False):
    return {"name": name, "kind": "norm", "T": T, "D": D, "x": x, "grad": grad}


def draw(rng) -> dict:
    """A case of the same kinds with sizes spread over their ranges."""
    cost = max(_cost(c) for c in listed())
    while True:
        case = _draw_once(rng)
        if _cost(case) <= cost and work(case)["bytes"] <= 4e9:
            del case["name"]
            return case


def _cost(case):
    """Seconds at nominal rates: what orders the cases by size."""
    w = work(case)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


def _between(rng, lo, hi, multiple=1):
    """A multiple of `multiple` in [lo, hi], uniform in the logarithm."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(x / multiple)) * multiple))


def _heads(rng):
    n_kv = rng.choice([1, 2, 4, 8, 16])
    return n_kv * rng.choice([1, 2, 4, 8] if n_kv <= 4 else [1, 2]), n_kv


def _draw_once(rng) -> dict:
    kind = rng.choice(["attention", "attention", "attention", "token", "token", "rope", "norm"])
    if kind == "attention":
        n_q, n_kv = _heads(rng)
        tokens = _between(rng, 200, 16384)
        causal = rng.random() < 0.75
        return _attention("", _between(rng, 1, max(1, tokens // 100)), tokens, n_q, n_kv, rng.choice([64, 64, 80, 96, 128, 128]), causal=causal,
                          prefix=_between(rng, 1, 1024) if causal and rng.random() < 0.3 else 0,
                          window=_between(rng, 64, 4096) if rng.random() < 0.3 else 0, cap=rng.choice([0.0, 30.0, 50.0]),
                          slopes=rng.random() < 0.3, grad=rng.random() < 0.7, fused=rng.random() < 0.5, cut=rng.randrange(1, 1000))
    if kind == "token":
        n_q, n_kv = _heads(rng)
        return _token("", _between(rng, 1, 128), _between(rng, 128, 16384, 64), n_q, n_kv, rng.choice([64, 80, 128, 128]),
                      window=_between(rng, 64, 4096) if rng.random() < 0.2 else 0, cap=rng.choice([0.0, 30.0, 50.0]),
                      slopes=rng.random() < 0.2, cut=rng.randrange(1, 1000))
    if kind == "rope":
        n_q, n_k = _heads(rng)
        dh = rng.choice([64, 80, 96, 128])
        rot = dh if rng.random() < 0.6 else dh // 2 // 16 * 16
        return _rope("", _between(rng, 1, 20000), n_q, n_k, dh, rot, rng.choice([1, 2, 3]), pairs=rng.random() < 0.5, inverse=rng.random() < 0.5,
                     far=rng.random() < 0.3)
    return _norm("", _between(rng, 1, 20000), _between(rng, 64, 8192, 8), x=rng.choice(["bf16", "bf16", "f32"]), grad=rng.random() < 0.6)


def _lengths(case):
    """Sequence lengths, a function of the case alone: ragged parts of the row, of which the last few tokens may belong to none."""
    rng = np.random.default_rng([case["cut"], case["n_seq"]])
    if case["kind"] == "token":                       # how far each request's cache is filled
        n = case["cache"] * rng.uniform(0.05, 1.0, case["n_seq"]) if case["n_seq"] > 1 else [0.7 * case["cache"]]
        return [max(1, int(x)) for x in n]
    if case["n_seq"] == 1:
        return [case["tokens"]]
    w = np.exp(rng.normal(0.0, 0.8, case["n_seq"]))
    used = case["tokens"] - min(case["tokens"] // 50, 37)
    return [max(1, int(x)) for x in used * w / w.sum()]


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def _pairs(case):
    """(query, allowed key) pairs of one head."""
    total = 0
    for n in _lengths(case):
        p = np.arange(n, dtype=np.int64) if case["kind"] == "attention" else np.array([n - 1], dtype=np.int64)
        lo, hi = np.zeros_like(p), np.full_like(p, n)
        if case.get("causal", True):
            hi = np.minimum(n, np.maximum(p + 1, case.get("prefix", 0)))
        if case["window"]:
            lo, hi = np.maximum(lo, p - case["window"] + 1), np.minimum(hi, p + case["window"])
        total += int((hi - lo).sum())
    return total


def work(case) -> dict:
    kind = case["kind"]
    if kind == "attention":
        rows = sum(_lengths(case))
        q, kv = rows * case["n_q"] * case["dh"] * 2, 2 * rows * case["n_kv"] * case["dh"] * 2
        # forward: q, k, v in, o out; backward: its gradient in, three gradients out (what the forward read is read once)
        return {"bytes": 2 * q + kv + (2 * q + kv if case["grad"] else 0),
                "flops": (14 if case["grad"] else 4) * case["dh"] * case["n_q"] * _pairs(case)}
    if kind == "token":
        return {"bytes": 2 * _pairs(case) * case["n_kv"] * case["dh"] * 2 + 2 * case["n_seq"] * case["n_q"] * case["dh"] * 2,
                "flops": 4 * case["dh"] * case["n_q"] * _pairs(case)}
    if kind == "rope":
        n = case["T"] * (case["n_q"] + case["n_k"])
        return {"bytes": 4 * n * case["dh"] + 4 * case["axes"] * case["T"], "flops": 3 * n * case["rot"]}
    n, x = case["T"] * case["D"], 2 if case["x"] == "bf16" else 4
    if not case["grad"]:
        return {"bytes": n * (x + 2) + 8 * case["D"], "flops": 7 * n}
    return {"bytes": n * (x + 2) + n * (6 + 2) + 16 * case["D"], "flops": 22 * n}


# ---- what a program holds before the call -----------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFFFFFF)


def _normal(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(torch.bfloat16)


def _slopes(n_q):
    """2^(-8 j / n_q), the usual geometric slopes of a distance bias."""
    return torch.tensor([2.0 ** (-8.0 * (j + 1) / n_q) for j in range(n_q)], dtype=torch.float32, device=DEV)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _with_outliers(t):
    """A few channels are larger than the rest, as in trained projections."""
    t[:, ::29] *= 4.0
    return t


def _inputs(case, seed):
    """The data of a case as a dict of tensors and plain values."""
    gen, kind = _generator(seed), case["kind"]
    if kind in ("attention", "token"):
        lens, n_q, n_kv, dh = _lengths(case), case["n_q"], case["n_kv"], case["dh"]
        tokens = case["tokens"] if kind == "attention" else case["n_seq"]
        keys = tokens if kind == "attention" else case["n_seq"] * case["cache"]
        starts = [sum(lens[:i]) for i in range(len(lens))] if kind == "attention" else [i * case["cache"] for i in range(case["n_seq"])]
        s = {"lens": lens, "starts": starts, "scale": dh ** -0.5, "slopes": _slopes(n_q) if case["slopes"] else None}
        widths = (n_q * dh, n_kv * dh, n_kv * dh)
        parts = [_with_outliers(_normal(gen, keys if i else tokens, w, scale=(1.7, 1.7, 1.0)[i])) for i, w in enumerate(widths)]
        if case.get("fused"):                             # one buffer, as a fused projection writes it
            whole = torch.cat(parts, dim=1)
            parts = list(whole.split(widths, dim=1))
        s["q"], s["k"], s["v"] = parts
        s["o"] = torch.zeros((tokens, widths[0]), dtype=torch.bfloat16, device=DEV)     # rows of no sequence stay as they are
        if case.get("grad"):
            s["d_o"] = _normal(gen, tokens, widths[0], scale=1e-2)
            grads = [torch.zeros((tokens, w), dtype=torch.bfloat16, device=DEV) for w in widths]
            s["grads"] = list(torch.cat(grads, dim=1).split(widths, dim=1)) if case["fused"] else grads
        return s
    if kind == "rope":
        T, half = case["T"], case["rot"] // 2
        edge = 1 << 20 if case["far"] else 512
        s = {"pos": torch.randint(0, edge, (case["axes"], T), generator=gen, device=DEV, dtype=torch.int32),
             "axis": [i * case["axes"] // half for i in range(half)], "freq": [THETA ** (-i / half) for i in range(half)]}
        s["q"] = _with_outliers(_normal(gen, T, case["n_q"] * case["dh"]))
        s["k"] = _with_outliers(_normal(gen, T, case["n_k"] * case["dh"]))
        return s
    T, D = case["T"], case["D"]
    x = torch.randn((T, D), generator=gen, device=DEV) + 0.5
    x[:, torch.randperm(D, generator=gen, device=DEV)[: max(1, D // 100)]] *= 30.0
    s = {"x": x if case["x"] == "f32" else x.to(torch.bfloat16), "g": torch.rand(D, generator=gen, device=DEV) + 0.5,
         "b": torch.randn(D, generator=gen, device=DEV) * 0.1}
    if case["grad"]:
        s["dh1"], s["dh2"], s["d_res"] = (_normal(gen, T, D, scale=1e-3) for _ in range(3))
    return s


def prepare(case, seed) -> dict:
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2603_22370_amd as faar
        s["faar"] = faar
        if case["kind"] in ("attention", "token"):
            # a mask's plan is made once for a batch (or a token) and read by all layers, forward and backward
            lens, starts = _ints(s["lens"]), _ints(s["starts"])
            token = case["kind"] == "token"
            prefix = _ints([case["prefix"]] * case["n_seq"]) if case.get("prefix") else None
            s["desc"] = faar.attention_description(case["n_q"], case["n_kv"], case["dh"], s["q"].shape[0], s["k"].shape[0], starts, lens,
                                                   single=token, prefix=prefix, window=case["window"], causal=case.get("causal", True),
                                                   scale=s["scale"], cap=case["cap"], slopes=s["slopes"])
            s["plan"] = faar.faar_attention_plan(s["desc"])
            s["ws"] = faar.attention_masked_workspace(s["desc"], backward=case.get("grad", False))
        if case["kind"] == "norm" and case["grad"]:
            s["ws"] = faar.layernorm_workspace(case["T"], case["D"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"attention": _own_attention, "token": _own_attention, "rope": _own_rope, "norm": _own_norm}[kind](s)
    return {"attention": _plain_attention, "token": _plain_attention, "rope": _plain_rope, "norm": _plain_norm}[kind](s)


def _own_attention(s):
    faar, grad = s["faar"], s["case"].get("grad", False)
    o, lse = faar.faar_attention_masked_fwd(s["desc"], s["plan"], s["q"], s["k"], s["v"], out=s["o"], want_lse=grad, ws=s["ws"])
    if not grad:
        return o
    dq, dk, dv = faar.faar_attention_masked_bwd(s["desc"], s["plan"], s["d_o"], s["q"], s["k"], s["v"], o, lse, out=s["grads"], ws=s["ws"])
    return {"o": o, "dq": dq, "dk": dk, "dv": dv}


def _own_rope(s):
    c = s["case"]
    return s["faar"].faar_rope_axes(s["q"], s["k"], c["n_q"], c["n_k"], c["dh"], s["pos"], s["axis"], s["freq"], pairs=c["pairs"],
                                    inverse=c["inverse"])


def _own_norm(s):
    faar, c = s["faar"], s["case"]
    h, mean, rstd = faar.faar_layernorm_fwd(s["x"], s["g"], s["b"], EPS)
    if not c["grad"]:
        return h
    dx, dg, db = faar.faar_layernorm_bwd(s["dh1"], s["x"], s["g"], mean, rstd, dh2=s["dh2"], d_res=s["d_res"], want_dg=True, want_db=True,
                                         ws=s["ws"])
    return {"h": h, "dx": dx, "dg": dg, "db": db}


def _plain_attention(s):
    """Sequence by sequence: scores, cap, bias, mask, softmax, product; then the same backwards.  float32 throughout."""
    c = s["case"]
    n_q, n_kv, dh, rep, token = c["n_q"], c["n_kv"], c["dh"], c["n_q"] // c["n_kv"], c["kind"] == "token"
    split = lambda t, h: t.float().view(t.shape[0], h, dh).transpose(0, 1).contiguous()                   # [heads, rows, dh]
    join = lambda t: t.transpose(0, 1).reshape(t.shape[1], -1).to(torch.bfloat16)
    for b, (at, n) in enumerate(zip(s["starts"], s["lens"])):
        rows = slice(b, b + 1) if token else slice(at, at + n)
        p = torch.arange(n - 1 if token else 0, n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None, :]
        seen = torch.ones((p.shape[0], n), dtype=torch.bool, device=DEV)
        if c.get("causal", True):
            seen &= (j <= p) | (j < c.get("prefix", 0))
        if c["window"]:
            seen &= (p - j).abs() < c["window"]
        k_all, v_all, q_all = split(s["k"][at:at + n], n_kv), split(s["v"][at:at + n], n_kv), split(s["q"][rows], n_q)
        o, grads = torch.empty_like(q_all), None
        if c.get("grad"):
            do_all = split(s["d_o"][rows], n_q)
            grads = [torch.empty_like(q_all), torch.zeros_like(k_all), torch.zeros_like(v_all)]
        for g in range(n_kv):                             # the query heads that share a key / value head
            h = slice(g * rep, (g + 1) * rep)
            kt, v = k_all[g].t().contiguous(), v_all[g]
            z = torch.matmul(q_all[h], kt) * s["scale"]
            if c["cap"]:
                th = torch.tanh(z / c["cap"])
                z = th * c["cap"]
            if s["slopes"] is not None:
                z = z - s["slopes"][h][:, None, None] * (p - j).abs()
            z = z.masked_fill(~seen, -math.inf)
            e = torch.exp(z - z.amax(dim=-1, keepdim=True))
            prob = e / e.sum(dim=-1, keepdim=True)
            o[h] = torch.matmul(prob, v)
            if grads is None:
                continue
            do = do_all[h]
            dp = torch.matmul(do, v.t().contiguous())
            ds = prob * (dp - (do * o[h]).sum(dim=-1, keepdim=True))
            if c["cap"]:
                ds = ds * (1.0 - th * th)
            ds = ds * s["scale"]
            grads[0][h] = torch.matmul(ds, k_all[g])
            grads[1][g] = torch.matmul(ds.flatten(0, 1).t(), q_all[h].flatten(0, 1))
            grads[2][g] = torch.matmul(prob.flatten(0, 1).t(), do.flatten(0, 1))
        s["o"][rows] = join(o)
        if grads is not None:
            for out, t in zip(s["grads"], grads):
                out[rows] = join(t)
    if not c.get("grad"):
        return s["o"]
    return {"o": s["o"], "dq": s["grads"][0], "dk": s["grads"][1], "dv": s["grads"][2]}


def _plain_rope(s):
    c = s["case"]
    half, dh = c["rot"] // 2, c["dh"]
    freq = torch.tensor(s["freq"], dtype=torch.float64, device=DEV)
    angle = s["pos"].double()[s["axis"]].t() * freq                                       # [T, half], 64 bits: positions are far
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin
    out = []
    for t in (s["q"], s["k"]):
        x = t.float().view(t.shape[0], -1, dh)
        y = x.clone()
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["pairs"] else (slice(0, half), slice(half, 2 * half))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        out.append(y.view_as(t).to(torch.bfloat16))
    return tuple(out)


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    d = x - mean
    r = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    xh = d * r
    h = (xh * s["g"] + s["b"]).to(torch.bfloat16)
    if not s["case"]["grad"]:
        return h
    dh = s["dh1"].float() + s["dh2"].float()
    gd = dh * s["g"]
    dx = r * (gd - gd.mean(dim=1, keepdim=True) - xh * (gd * xh).mean(dim=1, keepdim=True)) + s["d_res"].float()
    return {"h": h, "dx": dx.to(torch.bfloat16), "dg": (dh * xh).sum(dim=0), "db": dh.sum(dim=0)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"attention": _exact_attention, "token": _exact_attention, "rope": _exact_rope, "norm": _exact_norm}[case["kind"]](case, s)


def _exact_attention(c, s):
    """Head by head and a strip of queries at a time, log-sum-exp form; gradients by differentiation of the forward."""
    n_q, dh, token, grad = c["n_q"], c["dh"], c["kind"] == "token", c.get("grad", False)
    if (10 if grad else 4) * dh * n_q * sum(n * (1 if token else n) for n in s["lens"]) > 2.5e13:
        return None
    rep = n_q // c["n_kv"]
    q, k, v = (s[t].double() for t in "qkv")
    o = torch.zeros_like(q)
    do = s["d_o"].double() if grad else None
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v)) if grad else (None,) * 3
    for b, (at, n) in enumerate(zip(s["starts"], s["lens"])):
        keys = torch.arange(n, device=DEV, dtype=torch.float64)
        for head in range(n_q):
            cq, ck = slice(head * dh, (head + 1) * dh), slice(head // rep * dh, (head // rep + 1) * dh)
            slope = 2.0 ** (-8.0 * (head + 1) / n_q) if c["slopes"] else 0.0
            kh, vh = k[at:at + n, ck].detach(), v[at:at + n, ck].detach()
            first = n - 1 if token else 0
            for lo in range(first, n, 4096):
                hi = min(n, lo + 4096)
                rows = slice(b, b + 1) if token else slice(at + lo, at + hi)
                pos = torch.arange(lo, hi, device=DEV, dtype=torch.float64)
                gap = pos[:, None] - keys[None, :]
                hidden = torch.zeros_like(gap, dtype=torch.bool)
                if c.get("causal", True):
                    hidden |= (gap < 0) & (keys >= c.get("prefix", 0))[None, :]
                if c["window"]:
                    hidden |= gap.abs() >= c["window"]
                with torch.enable_grad():
                    leaves = [t.clone().requires_grad_(grad) for t in (q[rows, cq], kh, vh)]
                    z = leaves[0] @ leaves[1].T * s["scale"]
                    if c["cap"]:
                        z = c["cap"] * torch.tanh(z / c["cap"])
                    z = torch.where(hidden, torch.full_like(z, -math.inf), z - slope * gap.abs())
                    out = torch.exp(z - torch.logsumexp(z, dim=1, keepdim=True)) @ leaves[2]
                o[rows, cq] = out.detach()
                if grad:
                    got = torch.autograd.grad(out, leaves, do[rows, cq])
                    dq[rows, cq] = got[0]
                    dk[at:at + n, ck] += got[1]
                    dv[at:at + n, ck] += got[2]
    return {"o": o, "dq": dq, "dk": dk, "dv": dv} if grad else o


def _exact_rope(c, s):
    """The rotation as a product of complex numbers."""
    half = c["rot"] // 2
    sign = -1.0 if c["inverse"] else 1.0
    turn = torch.stack([s["pos"][s["axis"][i]].double() * (sign * s["freq"][i]) for i in range(half)], dim=1)
    turn = torch.polar(torch.ones_like(turn), turn)[:, None, :]
    out = []
    for t in (s["q"], s["k"]):
        x = t.double().view(c["T"], -1, c["dh"])
        y = x.clone()
        r = x[..., :2 * half]
        if c["pairs"]:
            y[..., :2 * half] = torch.view_as_real(torch.view_as_complex(r.reshape(*r.shape[:-1], half, 2).contiguous()) * turn).flatten(-2)
        else:
            w = torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous()) * turn
            y[..., :2 * half] = torch.cat([w.real, w.imag], dim=-1)
        out.append(y.view(c["T"], -1))
    return tuple(out)


def _exact_norm(c, s):
    """Gradients by differentiation of the forward."""
    grad = c["grad"]
    with torch.enable_grad():
        x, g, b = (s[t].double().requires_grad_(grad) for t in ("x", "g", "b"))
        mean = x.sum(dim=1, keepdim=True) / c["D"]
        var = ((x - mean) ** 2).sum(dim=1, keepdim=True) / c["D"]
        h = (x - mean) / torch.sqrt(var + EPS) * g + b
    if not grad:
        return h
    dx, dg, db = torch.autograd.grad(h, (x, g, b), s["dh1"].double() + s["dh2"].double())
    return {"h": h.detach(), "dx": dx + s["d_res"].double(), "dg": dg, "db": db}
