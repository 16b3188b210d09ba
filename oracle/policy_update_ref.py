"""fp64 references of the policy update's operators, written from their definitions (numpy, one head or row at a time).

Inputs are float arrays (bf16 data is widened by the caller).  Beside a gradient or a product the functions give the sum of the
magnitudes of its terms, from which the tests derive how far a result with 16-bit factors may be off.
"""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------- norm per head and rotation
def angles(positions, inv_freq, sections):
    """[T, d/2]: position on the axis of each frequency's section, times the frequency."""
    axis = np.repeat(np.arange(3), sections)
    return np.asarray(positions, np.float64)[axis].T * np.asarray(inv_freq, np.float64)


def _rotate(x, ang, sign):
    half = x.shape[-1] // 2
    z = (x[..., :half] + 1j * x[..., half:]) * np.exp(sign * 1j * ang)[:, None, :]
    return np.concatenate([z.real, z.imag], -1)


def norm_rope_ref(x, weight, positions, inv_freq, sections, eps):
    """x [T, H, d] -> y; weight None: rotation only."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    return _rotate(x, angles(positions, inv_freq, sections), 1)


def norm_rope_grad_ref(dy, x, weight, positions, inv_freq, sections, eps):
    """(dx, dweight, sum of |terms| of dweight)"""
    g = _rotate(np.asarray(dy, np.float64), angles(positions, inv_freq, sections), -1)
    if weight is None:
        return g, None, None
    x, w = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x / rms
    u = g * w
    return (u - n * (u * n).mean(-1, keepdims=True)) / rms, (g * n).sum((0, 1)), np.abs(g * n).sum((0, 1))


# ---------------------------------------------------------------- causal attention over packed sequences
def sequences(cu_seqlens, T):
    return [(a, b) for a, b in zip(cu_seqlens[:-1], cu_seqlens[1:]) if 0 <= a < b <= T]


def packed_attn_ref(q, k, v, cu_seqlens, scale):
    """q [T, Hq, d], k / v [T, Hkv, d] -> out [T, Hq, d], lse [Hq, T], sum of |terms| of out"""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, Hq, d = q.shape
    r = Hq // k.shape[1]
    out, mag, lse = np.zeros((T, Hq, d)), np.zeros((T, Hq, d)), np.full((Hq, T), -np.inf)
    for a, b in sequences(cu_seqlens, T):
        for h in range(Hq):
            for i in range(a, b):
                s = scale * (k[a:i + 1, h // r] @ q[i, h])
                m = s.max()
                e = np.exp(s - m)
                lse[h, i] = m + np.log(e.sum())
                p = e / e.sum()
                out[i, h] = p @ v[a:i + 1, h // r]
                mag[i, h] = p @ np.abs(v[a:i + 1, h // r])
    return out, lse, mag


def packed_attn_grad_ref(dout, q, k, v, cu_seqlens, scale, out_error=None):
    """dq, dk, dv and the sums of |terms| of each.  `out_error` [T, Hq, d]: how far the out that a row's sum of dout * out is
    taken from may be off; its effect is added to the magnitudes of dq and dk as if it were terms (divided by 2^-8)."""
    dout, q, k, v = (np.asarray(x, np.float64) for x in (dout, q, k, v))
    T, Hq, d = q.shape
    r = Hq // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    mq, mk, mv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for a, b in sequences(cu_seqlens, T):
        past = np.tril(np.ones((b - a, b - a), bool))
        for h in range(Hq):
            j = h // r
            Q, K, V, G = q[a:b, h], k[a:b, j], v[a:b, j], dout[a:b, h]
            s = np.where(past, scale * (Q @ K.T), -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            dp = G @ V.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            off = np.zeros((b - a, 1)) if out_error is None else (np.abs(G) * out_error[a:b, h]).sum(1, keepdims=True) * 256
            ads = np.abs(ds) + p * off
            dq[a:b, h] = scale * (ds @ K)
            dk[a:b, j] += scale * (ds.T @ Q)
            dv[a:b, j] += p.T @ G
            mq[a:b, h] = abs(scale) * (ads @ np.abs(K))
            mk[a:b, j] += abs(scale) * (ads.T @ np.abs(Q))
            mv[a:b, j] += p.T @ np.abs(G)
    return dq, dk, dv, mq, mk, mv


# ---------------------------------------------------------------- log-probs from hidden states
def linear_logprob_ref(hidden, weight, token_ids, inv_temperature=1.0):
    """logprob, lse, entropy [N]; a negative id: logprob 0, one past the vocabulary: NaN.  A logit that is -inf or NaN is masked."""
    z = (np.asarray(hidden, np.float64) @ np.asarray(weight, np.float64).T) * inv_temperature
    z = np.where(np.isnan(z), -np.inf, z)
    N, V = z.shape
    logprob, lse, entropy = np.zeros(N), np.zeros(N), np.zeros(N)
    for n in range(N):
        m = z[n].max()
        if np.isneginf(m):
            lse[n], entropy[n] = -np.inf, np.nan
            logprob[n] = 0.0 if token_ids[n] < 0 else (np.nan if token_ids[n] >= V else -np.inf)
            continue
        if np.isposinf(m):                                                    # no distribution either: not a number
            lse[n] = entropy[n] = np.nan
            logprob[n] = 0.0 if token_ids[n] < 0 else np.nan
            continue
        lse[n] = m + np.log(np.exp(z[n] - m).sum())
        lp = z[n] - lse[n]
        live = np.exp(lp) > 0
        entropy[n] = -(np.exp(lp[live]) * lp[live]).sum()
        y = token_ids[n]
        logprob[n] = 0.0 if y < 0 else (np.nan if y >= V else lp[y])
    return logprob, lse, entropy


def linear_logprob_grad_ref(hidden, weight, token_ids, g_logprob, g_entropy=None, inv_temperature=1.0):
    """dhidden, dweight and the sums of |terms| of each.  A row with no gradient of its own adds nothing, whatever it holds; dhidden sums
    over the columns whose dz is not 0, so that a masked token's weights do not reach it."""
    h, w = np.asarray(hidden, np.float64), np.asarray(weight, np.float64)
    N, V = h.shape[0], w.shape[0]
    dz = np.zeros((N, V))
    ge = np.zeros(N) if g_entropy is None else np.asarray(g_entropy, np.float64)
    for n in range(N):
        y = token_ids[n]
        gl = float(g_logprob[n]) if 0 <= y < V else 0.0
        if gl == 0.0 and ge[n] == 0.0:
            continue
        z = (w @ h[n]) * inv_temperature
        z = np.where(np.isnan(z), -np.inf, z)
        if np.isneginf(z.max()):
            continue
        lp = z - z.max()
        lp -= np.log(np.exp(lp).sum())
        p = np.exp(lp)
        flat = np.where(p > 0, lp, 0.0)
        ent = -(p * flat).sum()
        dz[n] = -gl * p - ge[n] * p * (flat + ent)
        if gl != 0.0:
            dz[n, y] += gl
        dz[n] *= inv_temperature
    used = np.abs(dz).max(1) > 0
    hu = h[used]
    finite = np.where(np.isfinite(w), w, 0.0)
    dh, mh = dz @ finite, np.abs(dz) @ np.abs(finite)
    for v in np.flatnonzero(~np.isfinite(w).all(1)):                          # of a masked token that was sampled
        rest = np.where(np.isfinite(w[v]), 0.0, w[v])
        for n in np.flatnonzero(dz[:, v]):
            dh[n, rest != 0] += dz[n, v] * rest[rest != 0]
    return dh, dz[used].T @ hu, mh, np.abs(dz[used]).T @ np.abs(hu)
