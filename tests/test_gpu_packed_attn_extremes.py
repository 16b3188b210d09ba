"""rl_packed_attn and its gradient where short sequences lie between long ones, at the ends of the range of scales and scores, next to NaN, and over very
many tokens.

Bars as in the parity tests (u = 2^-8, half a bf16 step at most): out 1.1 u (sum of |terms| + |out|) + 2e-5 of the terms; gradients the same of their
terms with 1e-4, D's error through out taken along as terms.
"""
import numpy as np
import pytest

from oracle import policy_update_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2512_21450_amd import binding
    return binding


def np64(t):
    return t.detach().double().cpu().numpy()


def inputs(T, Hq, Hkv, d, seed=0, gain=1.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    q, k, v, dout = (torch.randn(T, h, d, generator=g) for h in (Hq, Hkv, Hkv, Hq))
    return (q * gain).bfloat16().cuda(), k.bfloat16().cuda(), v.bfloat16().cuda(), dout.bfloat16().cuda()


def run(B, q, k, v, dout, cu, scale):
    import torch
    c = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out, lse = B.rl_packed_attn(q, k, v, c, scale)
    return (out, lse, *B.rl_packed_attn_backward(dout, q, k, v, out, lse, c, scale))


def check(got, q, k, v, dout, cu, scale, exponent=0.0):
    """exponent: how far a weight's exponent may be off beyond the parity tests' 1e-4"""
    out, lse, dq, dk, dv = (np64(t) for t in got)
    Q, K, V, G = (np64(t) for t in (q, k, v, dout))
    ro, rl, mo = R.packed_attn_ref(Q, K, V, cu, scale)
    bar = 1.1 * U * (mo + np.abs(ro)) + (2e-5 + exponent) * mo
    rq, rk, rv, mq, mk, mv = R.packed_attn_grad_ref(G, Q, K, V, cu, scale, out_error=bar)
    assert (np.abs(lse - rl) <= 2e-5 + 2e-7 * np.abs(rl) + exponent).all()
    for name, g, ref, tol in (("out", out, ro, bar), ("dq", dq, rq, 1.1 * U * (mq + np.abs(rq)) + (1e-4 + 2 * exponent) * mq),
                              ("dk", dk, rk, 1.1 * U * (mk + np.abs(rk)) + (1e-4 + 2 * exponent) * mk),
                              ("dv", dv, rv, 1.1 * U * (mv + np.abs(rv)) + (1e-4 + 2 * exponent) * mv)):
        assert np.isfinite(g).all(), name
        over = np.abs(g - ref) - tol
        assert (over <= 1e-30).all(), (name, np.unravel_index(over.argmax(), over.shape), np.abs(g - ref).max(), over.max())


@pytest.mark.parametrize("Hq,Hkv,d,lens", [(28, 4, 128, [1280, 3, 500, 9, 1, 700]), (14, 2, 64, [2, 300] * 12 + [5]), (8, 8, 128, [24, 100, 61, 340] * 3),
                                           (64, 8, 128, [1, 120] * 10), (6, 2, 64, [700, 20, 900, 15])])
def test_keys_of_few_rows_between_long_sequences(B, Hq, Hkv, d, lens):
    """A key that up to 64 rows see, and a row of up to 64 keys, takes along what rounding P and dS left over, whatever it is packed beside.  Bar as for
    short sequences alone: 2^-16 of each term, the result's own rounding 2^-8, exponents 1e-4, D 2^-16 of its terms."""
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    r, scale = Hq // Hkv, 1 / np.sqrt(d)
    x = inputs(cu[-1], Hq, Hkv, d, seed=Hq + d)
    got = [np64(t) for t in run(B, *x, cu, scale)[2:]]
    Q, K, V, G = (np64(t) for t in x)
    mo = R.packed_attn_ref(Q, K, V, cu, scale)[2]
    ref = R.packed_attn_grad_ref(G, Q, K, V, cu, scale, out_error=2.0 ** -11 * mo)
    few_rows = np.concatenate([(n - np.arange(n)) * r <= 64 for n in lens])
    few_keys = np.concatenate([np.arange(n) < 64 for n in lens])
    assert 0 < few_rows.sum() < cu[-1] and 0 < few_keys.sum() < cu[-1]
    for name, g, rr, m, at in zip(("dq", "dk", "dv"), got, ref[:3], ref[3:], (few_keys, few_rows, few_rows)):
        tol = 1.01 * U * np.abs(rr[at]) + (2.0 ** -15 + 1e-4) * m[at]
        off = np.abs(g[at] - rr[at])
        assert (off <= tol + 1e-30).all(), (name, (off / (tol + 1e-30)).max(), (off > tol + 1e-30).mean())


@pytest.mark.parametrize("Hq,Hkv,d,lens", [(4, 2, 128, [300]), (7, 1, 64, [20, 1, 190]), (3, 3, 128, [90, 64])])
def test_gradients_at_large_scores(B, Hq, Hkv, d, lens):
    """Scores up to some 100, sums of their terms' magnitudes up to M = some 300.  An exponent is a sum of d fp32 additions, each off by 2^-24 of the partial
    sum, from 0 on (out, dq) or from -lse / |scale| on (dk, dv): 4 * 2^-24 sqrt(d) (M + |lse|), and 4 * 2^-24 |lse| for the factors."""
    cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
    scale = 1 / np.sqrt(d)
    x = inputs(cu[-1], Hq, Hkv, d, seed=Hq, gain=25.0)
    got = run(B, *x, cu, scale)
    Q, K = np64(x[0]), np64(x[1])
    M = scale * max((np.abs(Q[:, h]) @ np.abs(K[:, h // (Hq // Hkv)]).T).max() for h in range(Hq))
    lse = np.abs(np64(got[1])).max()
    assert M < 1000 and lse > 50
    check(got, *x, cu, scale, exponent=4 * 2.0 ** -24 * (np.sqrt(d) * (M + lse) + lse))


@pytest.mark.parametrize("scale", [1e-29, 7e-31, -1e-33, 1e-36, 1e-38, -1e-38, 1e-42])
def test_scales_next_to_nothing(B, scale):
    """scores vanish: weights are equal, dv is their mean of dout; dq and dk vanish too"""
    cu = [0, 100, 101, 230]
    x = inputs(230, 4, 2, 64, seed=1)
    scale = float(np.float32(scale))
    check(run(B, *x, cu, scale), *x, cu, scale)


@pytest.mark.parametrize("power", [-122, -110, -102, -98, 60, 90])
def test_scales_that_make_up_for_the_inputs(B, power):
    """q and k of 2^-(power / 2): the same scores at any scale, and the same bits of out and lse"""
    import torch
    cu = [0, 100, 101, 230]
    q, k, v, dout = inputs(230, 4, 2, 64, seed=1)
    ref = run(B, q, k, v, dout, cu, 0.125)
    q2, k2 = (t.double().mul(2.0 ** (-power // 2)).bfloat16() for t in (q, k))
    got = run(B, q2, k2, v, dout, cu, 0.125 * 2.0 ** power)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    check((*got[:2], *((t.double() * 2.0 ** (-power // 2)) for t in got[2:4]), got[4]), q, k, v, dout, cu, 0.125)
