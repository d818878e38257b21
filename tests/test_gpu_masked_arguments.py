"""What the calls of layer norm, of the rotation over several axes and of attention under masks refuse among tensors that exist."""
import pytest
import torch

from test_gpu_masked_attention import ints

import paper_2603_22370_amd as faar


@pytest.mark.gpu
def test_rows_of_another_length_are_refused():
    """[D, T] where [T, D] is wanted has as many entries, and is not it."""
    T, D = 24, 64
    x, dh = (torch.randn(T, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    g = torch.ones(D, device="cuda")
    _, mean, rstd = faar.faar_layernorm_fwd(x, g)
    turned = dh.t().contiguous()
    dx, _, _ = faar.faar_layernorm_bwd(dh, x, g, mean, rstd)
    for kw in (dict(dh1=turned), dict(dh1=dh, dh2=turned), dict(dh1=dh, dh3=turned), dict(dh1=dh, d_res=turned)):
        with pytest.raises(ValueError, match="rows of 64"):
            faar.faar_layernorm_bwd(x=x, g=g, mean=mean, rstd=rstd, **kw)
    # rows in a shape of their own are rows all the same
    assert torch.equal(faar.faar_layernorm_bwd(dh.view(4, 6, D), x, g, mean, rstd)[0], dx)

    n_q, dh_ = 2, 64
    q, k, v, d_o = (torch.randn(T, n_q * dh_, device="cuda").to(torch.bfloat16) for _ in range(4))
    a = faar.attention_description(n_q, n_q, dh_, T, T, ints([0]), ints([T]))
    plan = faar.faar_attention_plan(a)
    o, stats = faar.faar_attention_masked_fwd(a, plan, q, k, v)
    for lse, low, width in ((stats.lse.t().contiguous(), stats.o_low, "rows of 24"), (stats.lse, stats.o_low.t().contiguous(), "rows of 128")):
        with pytest.raises(ValueError, match=width):
            faar.faar_attention_masked_bwd(a, plan, d_o, q, k, v, o, faar.AttentionStats(lse, low))


def test_lengths_of_their_own_for_caches_of_single_tokens_are_refused():
    n = torch.ones(2, dtype=torch.int32)
    for kw in (dict(k_start=n), dict(k_len=n), dict(k_start=n, k_len=n)):
        with pytest.raises(ValueError, match="those of the caches"):
            faar.attention_description(2, 1, 64, 2, 64, n, n, single=True, **kw)
