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


@pytest.mark.parametrize("Hq,Hkv,d,extra", [(4, 2, 128, 0), (4, 2, 64, 0), (4, 2, 128, 9000)])
def test_infinities_in_a_rows_own_range(B, Hq, Hkv, d, extra):
    """An infinite value makes its column of all rows that see it infinite, both kinds or a NaN make it NaN; an infinite dout the same of dv.  Everything else is
    what zeros in these places give.  (extra: so many tokens behind, which take a block of keys from several workgroups to one)"""
    import torch
    cu = [0, 40, 240] + ([240 + extra] if extra else [])
    T, scale = cu[-1], 0.09
    q, k, v, dout = inputs(T, Hq, Hkv, d, seed=d)
    x = [t.clone() for t in (q, k, v, dout)]
    inf, nan = float("inf"), float("nan")
    x[2][70, :, 5], x[2][100, :, 5], x[2][130, :, 7], x[2][60, 0, d - 1], x[2][150] = inf, -inf, nan, -inf, 0
    v[70, :, 5] = v[100, :, 5] = v[130, :, 7] = v[60, 0, d - 1] = v[150] = 0
    c = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out, lse = B.rl_packed_attn(*x[:3], c, scale)
    ref, rl, mag = R.packed_attn_ref(*(np64(t)[:240] for t in (q, k, v)), cu[:3], scale)
    want = ref.copy()
    want[70:100, :, 5], want[100:, :, 5], want[130:, :, 7], want[60:, :Hq // Hkv, d - 1] = inf, nan, nan, -inf
    got, fin = np64(out)[:240], np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    assert (np.abs(got - ref)[fin] <= (1.1 * U * (mag + np.abs(ref)) + 2e-5 * mag)[fin]).all()
    assert (np.abs(np64(lse)[:, :240] - rl) <= 2e-5 + 2e-7 * np.abs(rl)).all()
    # an infinite dout
    out, lse = B.rl_packed_attn(q, k, v, c, scale)
    dout[110, 0, 3] = dout[170, 1, 3] = dout[120, Hq - 1, 4] = 0
    x[3][:] = dout
    x[3][110, 0, 3], x[3][170, 1, 3], x[3][120, Hq - 1, 4] = inf, -inf, nan
    dq, dk, dv = (np64(t)[:240] for t in B.rl_packed_attn_backward(x[3], q, k, v, out, lse, c, scale))
    bar = 1.1 * U * (mag + np.abs(ref)) + 2e-5 * mag
    rq, _, rv, mq, _, mv = R.packed_attn_grad_ref(np64(dout)[:240], *(np64(t)[:240] for t in (q, k, v)), cu[:3], scale, out_error=bar)
    want = rv.copy()
    want[40:111, 0, 3], want[111:171, 0, 3], want[40:121, Hkv - 1, 4] = nan, -inf, nan             # up to 110: both infinities, of two heads
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(dv), np.isnan(want)) and np.array_equal(dv[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    assert (np.abs(dv - rv)[fin] <= (1.1 * U * (mv + np.abs(rv)) + 1e-4 * mv)[fin]).all()
    odd = np.zeros((240, Hq), bool)
    odd[110, 0] = odd[170, 1] = odd[120, Hq - 1] = True
    assert not np.isfinite(dq[odd]).any() and (np.abs(dq - rq)[~odd] <= (1.1 * U * (mq + np.abs(rq)) + 1e-4 * mq)[~odd]).all()
    seen = np.zeros((240, Hkv), bool)
    seen[40:171, 0] = seen[40:121, Hkv - 1] = True
    assert not np.isfinite(dk[seen]).any() and np.isfinite(dk[~seen]).all()


def times(f, n=5):
    import torch
    best = float("inf")
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("where", ["q", "k", "v", "kv"])
@pytest.mark.parametrize("token", [0, 2000, 5999])
def test_not_a_number_in_a_long_sequence(B, where, token):
    """NaN in one token of 6000: rows from it on are NaN (a query's own row alone), the others as ever; and a call takes the time of a few, not of a walk
    over the keys for every row"""
    import torch
    T, Hq, Hkv, d, scale = 6000, 7, 1, 128, 0.09
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    q, k, v, dout = inputs(T, Hq, Hkv, d, seed=2)
    ref = run(B, q, k, v, dout, [0, T], scale)

    def step():
        out, lse = B.rl_packed_attn(q, k, v, cu, scale)
        return (out, lse, *B.rl_packed_attn_backward(dout, q, k, v, out, lse, cu, scale))
    usual = times(step)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if name in where:
            t[token] = float("nan")
    out, lse, dq, dk, dv = step()
    rows = torch.zeros(T, dtype=torch.bool, device="cuda")
    rows[token:token + 1 if where == "q" else T] = True
    assert torch.isnan(out[rows].float()).all() and torch.isfinite(out[~rows].float()).all()
    assert (torch.isnan(lse[:, rows]).all() if where != "v" else torch.equal(lse, ref[1])) and torch.equal(lse[:, ~rows], ref[1][:, ~rows])
    assert ((out[~rows].float() - ref[0][~rows].float()).abs() <= 4 * U * ref[0][~rows].float().abs() + 2e-2).all()
    assert torch.isnan(dq[rows].float()).all() and torch.isfinite(dq[~rows].float()).all()
    assert ((dq[~rows].float() - ref[2][~rows].float()).abs() <= 4 * U * ref[2][~rows].float().abs() + 2e-2).all()
    # every key up to the last NaN row is seen by one
    last = token + 1 if where == "q" else T
    assert torch.isnan(dk[:last].float()).all() and torch.isfinite(dk[last:].float()).all() and torch.isfinite(dv[last:].float()).all()
    if where != "v":
        assert torch.isnan(dv[:last].float()).all()
    else:
        assert torch.equal(dv, ref[4])
    assert times(step) <= 10 * usual + 1.0


@pytest.mark.parametrize("d,T", [(64, 5), (128, 150), (128, 900)])
def test_scores_far_below_zero(B, d, T):
    """every score of a row near -1e32: the largest of them still is the row's reference"""
    import torch
    cu = [0, 3, T]
    q, k, v, dout = inputs(T, 4, 2, d, seed=d)
    q[:], k[:] = 2.0 ** 53, -2.0 ** 53
    out, lse = B.rl_packed_attn(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), 0.125)
    ref, rl, mag = R.packed_attn_ref(*(np64(t) for t in (q, k, v)), cu, 0.125)
    assert (np.abs(np64(lse) - rl) <= 1e-6 * np.abs(rl)).all()
    assert (np.abs(np64(out) - ref) <= 1.1 * U * (mag + np.abs(ref)) + 2e-5 * mag).all()


@pytest.mark.parametrize("T,r", [(300000, 1), (1 << 20, 2)])
def test_very_many_tokens_of_short_sequences(B, T, r):
    """sequences that repeat every 12800 tokens: gradients repeat to the bit, and are those of one call of 12800"""
    import torch
    n = 12800
    lens = [100, 1, 0, 37, 62] * 64
    assert sum(lens) == n
    q, k, v, dout = inputs(n, r, 1, 64, seed=3)
    cu = np.concatenate([[0], np.cumsum(lens)])
    ref = run(B, q, k, v, dout, cu.tolist(), 0.125)
    times = -(-T // n)
    many = np.concatenate([[0]] + [cu[1:] + n * i for i in range(times)])
    big = [t.repeat(times, 1, 1)[:T] for t in (q, k, v, dout)]
    got = run(B, *big, np.minimum(many, T).tolist(), 0.125)
    whole = T // n * n
    for g, c in zip((got[0], *got[2:]), (ref[0], *ref[2:])):
        assert torch.equal(g[:whole].view(-1, *c.shape), c.expand(T // n, *c.shape))
