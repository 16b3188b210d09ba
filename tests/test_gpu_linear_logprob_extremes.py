"""rl_linear_logprob and its gradient where weights are infinite or not numbers, and at the largest sizes that the header takes.

Bars are those of the parity tests: logits 8 * 2^-24 sqrt(H) max_v sum |h w| + 4 * 2^-24 |lse| (entropies and log-probs twice that); gradients
1.1 * 2^-8 (sum of |terms| + |result|) + 2 * the logits' bar * sum of |terms|.  Sums of magnitudes are taken over finite weights.
"""
import numpy as np
import pytest

from oracle import policy_update_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2512_21450_amd import binding
    return binding


def np64(t):
    return t.detach().double().cpu().numpy()


def inputs(N, H, V, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    h, w = torch.randn(N, H, generator=g).bfloat16().cuda(), (torch.randn(V, H, generator=g) * (2.5 / np.sqrt(H))).bfloat16().cuda()
    ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32).cuda()
    return h, w, ids, torch.randn(N, generator=g).cuda(), (0.3 * torch.randn(N, generator=g)).cuda()


def logit_bar(H, W, lse):
    """of rows with a distribution"""
    ok = np.isfinite(lse)
    W = np.where(np.isfinite(W), W, 0.0)
    return 8 * 2.0 ** -24 * np.sqrt(H.shape[1]) * (np.abs(H[ok]) @ np.abs(W).T).max() + 4 * 2.0 ** -24 * np.abs(lse[ok]).max()


# a tile of each form; columns that end inside a step of 64, and on its end
@pytest.mark.parametrize("N", [5, 60, 256, 300])
@pytest.mark.parametrize("H", [8, 64, 72, 200])
def test_infinite_weights_in_the_last_columns(B, N, H):
    """A logit of +inf leaves a row without a distribution (NaN), one of -inf or NaN masks its token, wherever among the columns the infinity lies"""
    h, w, ids, _, _ = inputs(N, H, 300, seed=N + H)
    w[17, H - 1] = float("inf")
    w[299, H - 1] = float("-inf")
    h[:, H - 1] = 0.0                                       # both tokens masked
    h[0::3, H - 1] = 1.0                                    # +inf, masked
    ids[1], ids[3] = 17, 17
    got = B.rl_linear_logprob(h, w, ids)
    H64, W64 = np64(h), np64(w)
    with np.errstate(all="ignore"):
        ref = dict(zip(("logprob", "lse", "entropy"), R.linear_logprob_ref(H64, W64, ids.cpu().numpy())))
    assert np.isnan(ref["lse"][0::3]).all() and np.isfinite(ref["lse"][1::3]).all()
    bar = logit_bar(H64, W64, ref["lse"])
    for name, r in ref.items():
        g = np64(got[name])
        assert np.array_equal(np.isnan(g), np.isnan(r)) and np.array_equal(np.isneginf(g), np.isneginf(r)), name
        f = np.isfinite(r)
        assert (np.abs(g[f] - r[f]) <= 2 * bar + 1e-6).all(), name


@pytest.mark.parametrize("N", [5, 300])
def test_masked_token_of_a_row_without_a_distribution(B, N):
    """next to a logit of +inf nothing has a log-prob, a masked token neither; without a live logit it is -inf"""
    import torch
    h, w, ids, _, _ = inputs(N, 64, 200, seed=N)
    h[:, 0] = 1.0
    w[:, 0] = 0.0
    w[7, 0], w[9, 0] = float("inf"), float("-inf")
    h[1::2, 0] = -1.0                                       # the two change places
    h[2] = float("nan")
    ids[0], ids[1], ids[2], ids[3] = 9, 7, 9, 5
    got = B.rl_linear_logprob(h, w, ids)
    with np.errstate(all="ignore"):
        ref = dict(zip(("logprob", "lse", "entropy"), R.linear_logprob_ref(np64(h), np64(w), ids.cpu().numpy())))
    assert np.isnan(ref["logprob"][[0, 1, 3]]).all() and np.isneginf(ref["logprob"][2])
    for name, r in ref.items():
        assert np.array_equal(np.isnan(np64(got[name])), np.isnan(r)) and np.array_equal(np.isneginf(np64(got[name])), np.isneginf(r)), name


@pytest.mark.parametrize("N,H,V", [(5, 64, 300), (40, 72, 129), (200, 136, 513), (256, 64, 300), (300, 264, 1000), (600, 64, 200)])
def test_masked_tokens_weights_reach_no_hidden_states_gradient(B, N, H, V):
    """Weights of -inf and NaN mask tokens.  dz is 0 there, and the sum over the vocabulary leaves them out: gradients are those of the weights with
    zeros in these places; a row without a gradient, or without a live logit, gets zeros.  A masked token that was sampled has a gradient, and passes on
    the infinity."""
    import torch
    h, w, ids, gl, ge = inputs(N, H, V, seed=N + H + V)
    h[:, H - 1] = 1.0
    w[:, H - 1] = 0.0
    w[10:90, H - 1] = float("-inf")                         # masks these tokens
    w[95] = float("nan")
    w[V - 1, H - 1] = float("-inf")                         # the last row, which the last tile reads again past the end
    ids[:] = torch.where((ids >= 10) & (ids < 100) | (ids == V - 1), 3, ids)
    ids[1], gl[1] = 20, 1.5                                 # a masked token was sampled
    gl[0] = ge[0] = 0
    ids[2], ge[2] = -1, 0
    h[3] = float("nan")                                     # no live logit
    got = B.rl_linear_logprob(h, w, ids)
    dh, dw = B.rl_linear_logprob_backward(h, w, ids, got["lse"], gl, entropy=got["entropy"], g_entropy=ge)
    H64, W64, y = np64(h), np64(w), ids.cpu().numpy()
    with np.errstate(all="ignore"):
        lse = R.linear_logprob_ref(H64, W64, y)[1]
        rh, rw, mh, mw = R.linear_logprob_grad_ref(H64, W64, y, np64(gl), np64(ge))
    assert np.isneginf(rh[1, H - 1]) and np.isfinite(np.delete(rh.ravel(), H + H - 1)).all() and np.isfinite(rw).all()
    assert (dh[0] == 0).all() and (dh[2] == 0).all() and (dh[3] == 0).all()
    assert np.isneginf(np64(dh)[1, H - 1])
    bar = logit_bar(H64, W64, lse)
    for name, g, ref, mag in (("dhidden", np64(dh), rh, mh), ("dweight", np64(dw), rw, mw)):
        f = np.isfinite(ref)
        assert np.isfinite(g[f]).all(), name
        assert (np.abs(g[f] - ref[f]) <= 1.1 * 2.0 ** -8 * (mag[f] + np.abs(ref[f])) + 2 * bar * mag[f] + 1e-30).all(), name


def test_masked_tokens_in_several_pieces(B):
    """20 thousand tokens: some 6.5 thousand columns of dz to a piece; masked tokens in the first and in the last one alone give zeros' gradients to the bit"""
    import torch
    N, H, V = 20000, 8, 15001
    h, w, ids, gl, ge = inputs(N, H, V, seed=3)
    ids[:] = ids.clamp(20, V - 20)
    for at in (slice(0, 9), slice(V - 9, V)):
        x, z = w.clone(), w.clone()
        x[at, :4] = float("nan")
        got = B.rl_linear_logprob(h, x, ids)
        dh, dw = B.rl_linear_logprob_backward(h, x, ids, got["lse"], gl, entropy=got["entropy"], g_entropy=ge)
        assert torch.isfinite(dh.float()).all() and torch.isfinite(dw.float()).all()
        p = h.float() @ w.float().T
        p[:, at] = -torch.inf
        lp = torch.log_softmax(p, -1)
        p = lp.exp()
        lp = lp.masked_fill(p == 0, 0.0)
        ent = -(p * lp).sum(-1)
        dz = -p * (gl[:, None] + ge[:, None] * (lp + ent[:, None]))
        dz.scatter_add_(1, ids.long()[:, None], gl[:, None])
        z[at] = 0
        for g, ref, mag in ((dh, dz @ z.float(), dz.abs() @ z.float().abs()), (dw, dz.T @ h.float(), dz.abs().T @ h.float().abs())):
            assert ((g.float() - ref).abs() <= 1.1 * 2.0 ** -8 * (mag + ref.abs()) + 1e-4 * mag).all()


def test_more_workgroups_than_one_dimension_of_a_grid_holds(B):
    """2^22 tokens over 2^17 + 300 of 8 columns: more than 2^32 threads of tiles.  Rows from all over against 64 bits."""
    import torch
    N, V, H = 1 << 22, (1 << 17) + 300, 8
    g = torch.Generator(device="cuda").manual_seed(0)
    h, w = (torch.randn(n, H, generator=g, device="cuda").bfloat16() for n in (N, V))
    ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32, device="cuda")
    got = B.rl_linear_logprob(h, w, ids)
    at = torch.tensor([0, 1, 255, 256, N // 2, (1 << 21) + 1, N - 257, N - 1], device="cuda")
    z = torch.stack([(w.double() * x).sum(1) for x in h[at].double()])
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    bar = 8 * 2.0 ** -24 * np.sqrt(H) * float((h[at].double().abs()[:, None] * w.double().abs()).sum(-1).max()) + 4 * 2.0 ** -24 * float(lse.abs().max())
    for name, ref, k in (("lse", lse, 1), ("logprob", lp.gather(1, ids[at].long()[:, None])[:, 0], 2), ("entropy", -(lp.exp() * lp).sum(1), 2)):
        assert ((got[name][at].double() - ref).abs() <= k * bar + 1e-6).all(), name
    assert torch.isfinite(got["lse"]).all() and torch.isfinite(got["entropy"]).all()


@pytest.mark.parametrize("N", [(1 << 24) - 70, 1 << 24])
def test_the_most_tokens(B, N):
    """2^24 tokens over 8 of 72 columns, with gradient: rows are those of a call of some of them"""
    import torch
    V, H = 8, 72
    g = torch.Generator(device="cuda").manual_seed(0)
    h, w = (torch.randn(n, H, generator=g, device="cuda").bfloat16() for n in (N, V))
    ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32, device="cuda")
    gl = torch.zeros(N, device="cuda")
    # 256 tokens, in one tile and from all over, have gradients: dweight is theirs
    at = torch.cat([torch.arange(0, 64), torch.arange(1 << 23, (1 << 23) + 64), torch.arange(N - 128, N)]).cuda()
    gl[at] = torch.randn(256, generator=g, device="cuda")
    got = B.rl_linear_logprob(h, w, ids)
    dh, dw = B.rl_linear_logprob_backward(h, w, ids, got["lse"], gl)
    ref = B.rl_linear_logprob(h[at], w, ids[at])
    rh, rw = B.rl_linear_logprob_backward(h[at], w, ids[at], ref["lse"], gl[at])
    assert all(torch.equal(got[k][at], ref[k]) for k in got)
    mag = dh[at].float().abs() + rh.float().abs()
    assert ((dh[at].float() - rh.float()).abs() <= 2.0 ** -7 * mag).all() and dh[at].abs().max() > 0.1        # a rounding of each
    idle = torch.ones(N, dtype=torch.bool, device="cuda")
    idle[at] = False
    assert (dh[idle] == 0).all()
    z = h[at].double() @ w.double().T.contiguous()
    dz = -z.softmax(1)
    dz[torch.arange(256), ids[at].long()] += 1
    dz *= gl[at].double()[:, None]
    rw, mw = dz.T.contiguous() @ h[at].double(), dz.abs().T.contiguous() @ h[at].double().abs()
    assert ((dw.double() - rw).abs() <= 1.1 * 2.0 ** -8 * (mw + rw.abs()) + 1e-4 * mw).all()


def test_the_largest_vocabulary_without_tokens(B):
    import torch
    w = torch.ones(1 << 24, 8, dtype=torch.bfloat16, device="cuda")
    h, ids, f = torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    dw = torch.ones_like(w)
    B.rl_linear_logprob_backward(h, w, ids, f, f, want=(), dweight=dw)
    assert (dw == 0).all()
