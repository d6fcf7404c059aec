"""Causal attention with a sliding window and sinks over packed segments, fp64 (test infrastructure).

Token i of a segment sees its token j iff j <= i and (i - j < window or j < sinks); everything else is the
definition of ``oracle.attention``.  One dense mask a segment and head: small segments only, besides
``rows``, which evaluates chosen rows.
"""
from __future__ import annotations

import math

import numpy as np

from .attention import _f64, kv_head


def visible(i, j, window, sinks):
    """Of positions in a segment (arrays broadcast)."""
    return (j <= i) & ((i - j < window) | (j < sinks))


def _scale(scale, d):
    return 1.0 / math.sqrt(d) if scale is None or scale <= 0 else float(scale)


def attn(q, k, v, cu_seqlens, window, sinks=0, do=None, scale=None):
    """dict of o [N, Hq, d] and lse [Hq, N], and with do also dq, dk, dv.  ``p`` and ``ds`` list, segment by
    segment and head by head, what error bounds are made of: (segment, head, P, dS, dP, D)."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    do = None if do is None else _f64(do)
    n, hq, d = q.shape
    hkv = k.shape[1]
    scale = _scale(scale, d)
    out = dict(o=np.zeros_like(q), lse=np.zeros((hq, n)), parts=[])
    if do is not None:
        out.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v))
    cu = [int(x) for x in cu_seqlens]
    for b, e in zip(cu[:-1], cu[1:]):
        pos = np.arange(e - b)
        seen = visible(pos[:, None], pos[None, :], window, sinks)
        for h in range(hq if e > b else 0):
            g = kv_head(h, hq, hkv)
            qh, kh, vh = q[b:e, h], k[b:e, g], v[b:e, g]
            s = np.where(seen, scale * (qh @ kh.T), -np.inf)
            m = s.max(axis=1, keepdims=True)
            lse = m + np.log(np.exp(s - m).sum(axis=1, keepdims=True))
            p = np.exp(s - lse)
            o = p @ vh
            out["o"][b:e, h], out["lse"][h, b:e] = o, lse[:, 0]
            if do is None:
                out["parts"].append((b, e, h, g, p, None, None, None))
                continue
            dh = do[b:e, h]
            dp = np.where(seen, dh @ vh.T, 0.0)
            dd = (dh * o).sum(axis=1, keepdims=True)
            ds = p * (dp - dd)
            out["dq"][b:e, h] = scale * (ds @ kh)
            out["dk"][b:e, g] += scale * (ds.T @ qh)
            out["dv"][b:e, g] += p.T @ dh
            out["parts"].append((b, e, h, g, p, ds, dp, dd))
    return out


def rows(q, k, v, seg, h, positions, window, sinks=0, scale=None):
    """(o [len, d], lse [len]) of chosen rows of one segment (b, e) and head."""
    b, _ = seg
    g = kv_head(h, q.shape[1], k.shape[1])
    scale = _scale(scale, q.shape[-1])
    o, lse = [], []
    for i in positions:
        j = np.concatenate([np.arange(min(sinks, max(0, i - window + 1))), np.arange(max(0, i - window + 1), i + 1)])
        s = scale * (_f64(k[b + j, g]) @ _f64(q[b + i, h]))
        m = s.max()
        lse.append(m + np.log(np.exp(s - m).sum()))
        o.append(np.exp(s - lse[-1]) @ _f64(v[b + j, g]))
    return np.array(o), np.array(lse)
