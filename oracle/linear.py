"""Linear attention with a decay for each key/value head, fp64 (test infrastructure).

Over the tokens of a segment, with lam = exp(log_decay) of the head and query heads in contiguous groups:

  S_t = lam S_{t-1} + k_t v_t^T (S before the first token given or 0),   o_t = scale q_t^T S_t

`walk` is that recurrence, token by token.  `attn` and `grads` are the sums it stands for,
o_t = scale (lam^(t+1) q_t S + sum_{s <= t} lam^(t-s) (q_t . k_s) v_s), and their derivatives.
"""
from __future__ import annotations

import numpy as np


def _f64(x):
    return np.asarray(x.double().cpu().numpy() if hasattr(x, "cpu") else x, dtype=np.float64)


def _scale(scale, d):
    return scale if scale > 0 and np.isfinite(scale) else 1.0 / np.sqrt(d)


def walk(q, k, v, log_decay, cu, state=None, scale=0.0):
    """(o, states behind the segments)."""
    q, k, v, g = _f64(q), _f64(k), _f64(v), _f64(log_decay)
    (n, hq, d), hkv = q.shape, k.shape[1]
    cu = np.asarray(cu, np.int64)
    o, out = np.zeros_like(q), np.zeros((len(cu) - 1, hkv, d, d))
    for s, (b, e) in enumerate(zip(cu[:-1], cu[1:])):
        st = np.zeros((hkv, d, d)) if state is None else _f64(state[s]).copy()
        for t in range(b, e):
            for h in range(hkv):
                st[h] = np.exp(g[h]) * st[h] + np.outer(k[t, h], v[t, h])
            for h in range(hq):
                o[t, h] = _scale(scale, d) * (q[t, h] @ st[h * hkv // hq])
        out[s] = st
    return o, out


def weights(n, g):
    """[n, n]: lam^(t-s) for s <= t, else 0."""
    gap = np.arange(n)[:, None] - np.arange(n)[None]
    return np.where(gap >= 0, np.exp(g * np.maximum(gap, 0)), 0.0)


def attn(q, k, v, log_decay, cu, state=None, scale=0.0):
    """dict of o, the states behind the segments, and the same sums over absolute values (o_abs, states_abs)."""
    q, k, v, g = _f64(q), _f64(k), _f64(v), _f64(log_decay)
    (n, hq, d), hkv = q.shape, k.shape[1]
    cu, sc = np.asarray(cu, np.int64), _scale(scale, q.shape[2])
    o, oa = np.zeros_like(q), np.zeros_like(q)
    st = np.zeros((len(cu) - 1, hkv, d, d)) if state is None else _f64(state).copy()
    sa = np.abs(st)
    for s, (b, e) in enumerate(zip(cu[:-1], cu[1:])):
        for h in range(hkv):
            w = weights(e - b, g[h])
            for x in range(h * hq // hkv, (h + 1) * hq // hkv):
                far = np.exp(g[h] * np.arange(1, e - b + 1))[:, None]
                o[b:e, x] = sc * (far * (q[b:e, x] @ st[s, h]) + (w * (q[b:e, x] @ k[b:e, h].T)) @ v[b:e, h])
                oa[b:e, x] = sc * (far * (np.abs(q[b:e, x]) @ sa[s, h])
                                   + (w * (np.abs(q[b:e, x]) @ np.abs(k[b:e, h]).T)) @ np.abs(v[b:e, h]))
            left = np.exp(g[h] * np.arange(e - b - 1, -1, -1))[:, None]
            fade = np.exp(g[h] * (e - b)) if e > b else 1.0
            st[s, h] = fade * st[s, h] + (left * k[b:e, h]).T @ v[b:e, h]
            sa[s, h] = fade * sa[s, h] + (left * np.abs(k[b:e, h])).T @ np.abs(v[b:e, h])
    return dict(o=o, state=st, o_abs=oa, state_abs=sa)


def grads(q, k, v, dout, log_decay, cu, scale=0.0):
    """dict of dq, dk, dv of `attn` without a state, and the sums over absolute values (dq_abs, dk_abs, dv_abs)."""
    q, k, v, do, g = _f64(q), _f64(k), _f64(v), _f64(dout), _f64(log_decay)
    (n, hq, d), hkv = q.shape, k.shape[1]
    cu, sc = np.asarray(cu, np.int64), _scale(scale, q.shape[2])
    r = {a + b: np.zeros_like(x) for a, x in (("dq", q), ("dk", k), ("dv", v)) for b in ("", "_abs")}
    for b, e in zip(cu[:-1], cu[1:]):
        for x in range(hq):
            h = x * hkv // hq
            w = sc * weights(e - b, g[h])
            for tail, f in (("", lambda y: y), ("_abs", np.abs)):
                qx, kx, vx, dx = f(q[b:e, x]), f(k[b:e, h]), f(v[b:e, h]), f(do[b:e, x])
                p, ds = w * (qx @ kx.T), w * (dx @ vx.T)
                r["dq" + tail][b:e, x] = ds @ kx
                r["dk" + tail][b:e, h] += ds.T @ qx
                r["dv" + tail][b:e, h] += p.T @ dx
    return r


def row(q, k, v, g, b, t, x, h, scale=0.0):
    """o of token t of the segment that starts at b, query head x, key/value head h of decay g; and its absolute sum."""
    j = np.arange(b, t + 1)
    w = np.exp(float(g) * (t - j))
    qt, kj, vj = _f64(q[t, x]), _f64(k[b:t + 1, h]), _f64(v[b:t + 1, h])
    sc = _scale(scale, q.shape[2])
    return sc * (w * (kj @ qt)) @ vj, sc * (w * (np.abs(kj) @ np.abs(qt))) @ np.abs(vj)
