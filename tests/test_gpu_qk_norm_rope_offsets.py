"""rl_qk_norm_rope over more tokens than one dimension of a grid has workgroups for."""
import pytest

pytestmark = pytest.mark.gpu


def test_more_than_2_26_tokens():
    """2^26 + 5 tokens of one head each, forward and gradient, the latter in place: tokens from all over are those of a small call, to the bit"""
    import torch
    from paper_2512_21450_amd import binding as B
    T, d = (1 << 26) + 5, 64
    g = torch.Generator(device="cuda").manual_seed(0)
    at = torch.cat([torch.arange(0, 2000), torch.arange(1 << 25, (1 << 25) + 64), torch.arange((1 << 26) - 64, T)]).cuda()
    few = [torch.randn(len(at), 1, d, generator=g, device="cuda").bfloat16() for _ in range(2)]
    x = [torch.zeros(T, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    x[0][at], x[1][at] = few
    pos = torch.randint(0, 40000, (3, T), generator=g, device="cuda", dtype=torch.int32)
    freq = torch.logspace(0, -6, d // 2).cuda()
    qw, kw = (torch.randn(d, generator=g, device="cuda") for _ in range(2))
    args = (freq, (8, 12, 12), qw, kw, 1e-6)
    q, k = B.rl_qk_norm_rope(*x, pos, *args)
    ref = B.rl_qk_norm_rope(*few, pos[:, at].contiguous(), *args)
    assert torch.equal(q[at], ref[0]) and torch.equal(k[at], ref[1]) and ref[0].abs().max() > 0.1
    B.rl_qk_norm_rope_backward(q, k, *x, pos, *args, dq=q, dk=k)
    ref = B.rl_qk_norm_rope_backward(*ref, *few, pos[:, at].contiguous(), *args)
    assert torch.equal(q[at], ref[0]) and torch.equal(k[at], ref[1])
