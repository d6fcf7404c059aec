"""Rotary positions with several axes over training segments, fp64 (test infrastructure).

The paper's path applies no positions.  What is computed here: a segment's tokens are walked in order
with a running position p; a text token stands at (p, p, p) and moves p by one, a screenshot of T x H x W
tokens puts its token (t, y, x) at (p + t, p + y, p + x) and moves p by max(T, H, W).  Pair i of a head,
dims (a, b), is turned by inv_freq[i] * (position on axis pair_axis[i]):

  (a, b) -> (a cos - b sin, b cos + a sin)

and the gradient of a trajectory row is the sum over its segment copies of their gradients turned back
(the transpose of the rotation composed with the copy).
"""
from __future__ import annotations

import numpy as np


def _f64(x):
    if hasattr(x, "detach"):
        return x.detach().to("cpu").double().numpy()
    return np.asarray(x, dtype=np.float64)


def positions(cu_seqlens, tok_src_step, step_img, step_txt, step_grid):
    """int64 [3, N], token by token."""
    cu, src = np.asarray(cu_seqlens), np.asarray(tok_src_step)
    pos = np.zeros((3, len(src)), np.int64)
    for b, e in zip(cu[:-1], cu[1:]):
        p, n = 0, int(b)
        while n < e:
            s = int(src[n])
            run = 0
            while n + run < e and src[n + run] == s:
                run += 1
            if run == step_img[s] + step_txt[s]:          # the screenshot is there too
                t, h, w = (int(x) for x in step_grid[s])
                for k, (z, y, x) in enumerate(np.ndindex(t, h, w)):
                    pos[:, n + k] = (p + z, p + y, p + x)
                n, run = n + t * h * w, run - t * h * w
                p += max(t, h, w) if t * h * w else 0
            for k in range(run):
                pos[:, n + k] = p + k
            n, p = n + run, p + run
    return pos


def frequencies(rot_dim, sections, theta):
    """(inv_freq, pair_axis) with axis a taking the next sections[a] pairs."""
    inv = [theta ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    return np.array(inv), np.repeat(np.arange(len(sections)), sections)


def rotate(x, pos, inv_freq, pair_axis, interleaved=False, back=False):
    """x [N, heads, d] turned by pos [axes, N]; dims from 2 * len(inv_freq) on unchanged."""
    y, half = _f64(x).copy(), len(inv_freq)
    pos = np.asarray(pos, np.float64)
    for i in range(half):
        ang = (inv_freq[i] * pos[pair_axis[i]])[:, None] * (-1 if back else 1)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        u, v = y[..., a].copy(), y[..., b].copy()
        y[..., a] = u * np.cos(ang) - v * np.sin(ang)
        y[..., b] = v * np.cos(ang) + u * np.sin(ang)
    return y


def inverse(tok_gather, traj_tokens):
    """(off, tok): the segment tokens of each trajectory token, in order."""
    lists = [[] for _ in range(traj_tokens)]
    for n, t in enumerate(np.asarray(tok_gather)):
        if 0 <= t < traj_tokens:
            lists[t].append(n)
    return (np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int64),
            np.array([n for x in lists for n in x], np.int64))


def scatter(x, tok_gather, traj_tokens):
    """Sum of segment rows over each trajectory token's copies."""
    out = np.zeros((traj_tokens,) + x.shape[1:])
    np.add.at(out, np.asarray(tok_gather), x)
    return out
