"""Rotary positions with several axes and windowed attention over training segments, as timed cases.

A training program cuts trajectories of screenshots and responses into segments, gives every segment
token a position on three axes (time, height, width), gathers the packed rows of Q, K and V with the
rotation applied, runs attention that sees the last `window` tokens and the first `sinks` tokens of
the segment, and takes the gradients back to the trajectory's rows.  Each case is one of these:

  layout   positions of a layout's tokens, and the inverse of its gather map (once per batch)
  rope     Q, K, V of the segments from trajectory rows, rotated
  unrope   gradients of the trajectory rows from the segments' (rotated back, summed over copies)
  fwd      windowed attention, output and log-sum-exp (scoring, reference policy)
  train    the same and its gradients

Where `own` is false they are computed by elementary torch operations in 32 bits (angles in 64).
The step counts that fix a case's shapes come from its own `shape` number, the tensors from the seed.
"""
import functools
import math

import numpy as np
import torch

own = False
DEV = "cuda"


def _case(name, kind, traj, steps, rows, cols, txt, cut, keep, heads, window=0, sinks=0, frames=1, interleaved=False,
          shape=1):
    return dict(name=name, kind=kind, traj=traj, steps_lo=steps[0], steps_hi=steps[1], rows_lo=rows[0], rows_hi=rows[1],
                cols_lo=cols[0], cols_hi=cols[1], txt_lo=txt[0], txt_hi=txt[1], frames=frames, cut=cut, keep=keep,
                hq=heads[0], hkv=heads[1], d=heads[2], window=window, sinks=sinks, interleaved=interleaved, shape=shape)


TINY = ((4, 4), (16, 16), (16, 16), (32, 32))         # a four-step rollout of 256-token screenshots
SHORT = ((5, 15), (32, 32), (32, 32), (64, 256))      # short rollouts, 1,024-token screenshots
MIXED = ((10, 30), (30, 45), (50, 60), (64, 512))     # screenshots of 1,500 to 2,700 tokens
LONG = ((50, 50), (45, 45), (60, 60), (512, 512))     # long-horizon rollouts, 2,700-token screenshots


def listed():
    return [
        # the layout of one four-step rollout: launches and latency
        _case("layout_tiny", "layout", 1, (4, 4), (8, 8), (32, 32), (32, 32), 2, 0, (2, 1, 64)),
        # the layout of a collection of long rollouts at once (15.8 M segment tokens)
        _case("layout_batch", "layout", 64, *LONG, 8, 0, (40, 8, 128)),
        # the rotated rows of one four-step rollout: latency
        _case("rope_tiny", "rope", 1, *TINY, 2, 0, (2, 1, 64)),
        # the rotated rows of one long rollout, at the largest row size
        _case("rope_long", "rope", 1, *LONG, 8, 0, (40, 8, 128)),
        # the gradients' way back for short rollouts of 64-wide heads, one screenshot retained, neighbouring pairs
        _case("unrope_d64", "unrope", 8, *SHORT, 3, 1, (14, 2, 64), interleaved=True, shape=2),
        # and for one long rollout
        _case("unrope_long", "unrope", 1, *LONG, 8, 0, (40, 8, 128)),
        # scoring of one four-step rollout with a short window: latency
        _case("fwd_tiny", "fwd", 1, *TINY, 2, 0, (2, 1, 64), 128, 4),
        # scoring of a batch of short rollouts, an ordinary window
        _case("fwd_short", "fwd", 8, *SHORT, 3, 0, (28, 4, 128), 1024, 4, shape=2),
        # scoring of one long rollout, whose segments of 25,696 to 46,176 tokens are many windows long
        _case("fwd_long", "fwd", 1, *LONG, 8, 0, (40, 8, 128), 2048, 64),
        # the actor update of a batch of short rollouts with 64-wide heads, an odd window
        _case("train_d64", "train", 8, *SHORT, 3, 0, (14, 2, 64), 511, 16, shape=2),
        # the actor update of a few full-screen rollouts, no sinks, the shortest ordinary window
        _case("train_mixed", "train", 2, *MIXED, 3, 0, (28, 4, 128), 256, 0, shape=6),
        # the actor update of one long rollout
        _case("train_long", "train", 1, *LONG, 8, 0, (40, 8, 128), 1024, 4),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["layout", "rope", "unrope", "fwd", "fwd", "train", "train"])
    heads = rng.choice([(2, 1, 64), (4, 4, 64), (14, 2, 64), (6, 2, 128), (16, 2, 128), (28, 4, 128), (40, 8, 128)])
    window, sinks = log(32, 4096), rng.choice([0, 1, 4, rng.randrange(2, 65), 128])
    # tokens of the layout: up to what the largest listed case of the kind costs
    wide = heads[0] * heads[2] * (window + sinks + 128)
    most = dict(layout=12e6, rope=2e9 / (heads[0] * heads[2]), unrope=2e9 / (heads[0] * heads[2]),
                fwd=3e12 / wide, train=1.5e12 / wide)[kind]
    tokens = log(600, max(1200, min(most, 12e6 if kind == "layout" else 250_000)))
    rows, cols, txt = rng.randrange(8, 46), rng.randrange(8, 61), rng.randrange(1, 500)
    cut, keep = rng.randrange(1, 9), rng.randrange(0, 3)
    step = rows * cols * 0.8 + txt * 0.6
    steps = 2  # as many steps a rollout, up to 50, as keep two rollouts' segments within the tokens
    while steps < 50 and 2 * (steps + 1) * step * (1 + keep / cut) * (1 + (steps + 1) * 0.1 / cut) < tokens:
        steps += 1
    per = steps * step * (1 + keep / cut) * (1 + steps * 0.1 / cut)
    return _case(None, kind, max(1, min(512, int(tokens / per))), (max(1, steps // 2), steps),
                 (max(1, rows // 2), rows), (max(1, cols // 2), cols), (0, txt), cut, keep, heads,
                 window if kind in ("fwd", "train") else 0, sinks if kind in ("fwd", "train") else 0,
                 frames=rng.choice([1, 1, 2]), interleaved=rng.random() < 0.3,
                 shape=rng.randrange(1, 1 << 20)) | ({} if kind in ("fwd", "train") else {"sinks": 0})


# ------------------------------------------------------------------ inputs

def _layout(c, seed=None):
    """Steps and segment layout of a case as numpy arrays.  A seed turns some screenshots on their side."""
    return _layout_of(c["shape"], seed, c["traj"], c["steps_lo"], c["steps_hi"], c["rows_lo"], c["rows_hi"],
                      c["cols_lo"], c["cols_hi"], c["txt_lo"], c["txt_hi"], c["frames"], c["cut"], c["keep"])


@functools.lru_cache(maxsize=4)
def _layout_of(shape, seed, traj, s0, s1, r0, r1, c0, c1, t0, t1, frames, cut, keep):
    rng = np.random.default_rng(shape)
    counts = rng.integers(s0, s1, size=traj, endpoint=True)
    n = int(counts.sum())
    rows, cols = rng.integers(r0, r1, size=n, endpoint=True), rng.integers(c0, c1, size=n, endpoint=True)
    grid = np.stack([rng.integers(1, frames, size=n, endpoint=True), rows, cols], 1).astype(np.int32)
    txt = rng.integers(t0, t1, size=n, endpoint=True).astype(np.int32)
    ends = np.cumsum(counts)
    if seed is not None:
        side = np.random.default_rng(seed).random(n) < 0.5
        grid[side, 1:] = grid[side, :0:-1]
    img = grid.prod(1).astype(np.int32)
    base = np.concatenate([[0], np.cumsum(img.astype(np.int64) + txt)])
    first, length, step, seg_runs = [], [], [], []
    for e, m in zip(ends, counts):
        b, done, stop = int(e - m), 0, min(int(m), keep + cut)
        while m:
            s = np.arange(b, b + stop)
            whole = np.arange(stop) >= done - keep      # steps before keep their text only
            first.append(base[s] + np.where(whole, 0, img[s]))
            length.append(txt[s] + np.where(whole, img[s], 0))
            step.append(s)
            seg_runs.append(stop)
            if stop == m:
                break
            done, stop = stop, min(int(m), stop + cut)
    first, length, step = (np.concatenate(x).astype(np.int64) for x in (first, length, step))
    at = np.concatenate([[0], np.cumsum(length)])
    cu = at[np.concatenate([[0], np.cumsum(seg_runs)])]
    gather = np.repeat(first - at[:-1], length) + np.arange(at[-1])
    return dict(cu=cu.astype(np.int32), gather=gather.astype(np.int32), src=np.repeat(step, length).astype(np.int32),
                img=img, txt=txt, grid=grid, traj_tokens=int(base[-1]), tokens=int(at[-1]),
                longest=int(np.diff(cu).max()))


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _sections(d):
    return (16, 24, 24) if d == 128 else (8, 12, 12)


THETA = 1e6


def prepare(case, seed):
    lay = _layout(case, seed if case["kind"] == "layout" else None)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, hq, hkv, d = (case[k] for k in ("kind", "hq", "hkv", "d"))
    n, t = lay["tokens"], lay["traj_tokens"]
    s = dict(case=case, tokens=n, traj_tokens=t, longest=lay["longest"])
    for key in ("cu", "gather", "src", "img", "txt", "grid"):
        s[key] = torch.from_numpy(lay[key]).to(DEV)
    if kind in ("rope", "unrope"):
        # what a training loop made once for the layout: the positions and the inverse map
        s["pos"] = _positions(s)
        s["inv"] = _inverse(s)
    rows = t if kind == "rope" else n
    if kind != "layout":
        s["q"], s["k"], s["v"] = _normal(gen, rows, hq, d), _normal(gen, rows, hkv, d), _normal(gen, rows, hkv, d)
    if kind == "train":
        s["do"] = _normal(gen, n, hq, d)
    return s


# ------------------------------------------------------------------ plain forms

def _positions(s):
    """Positions [3, tokens] int32: a run is one step's tokens in one segment."""
    src, cu, grid = s["src"].long(), s["cu"].long(), s["grid"].long()
    n = torch.arange(s["tokens"], device=DEV)
    seg = torch.searchsorted(cu[1:], n, right=True)
    new = torch.ones_like(n, dtype=torch.bool)
    new[1:] = (src[1:] != src[:-1]) | (seg[1:] != seg[:-1])
    run = torch.cumsum(new, 0) - 1
    at = torch.nonzero(new)[:, 0]
    length = torch.diff(at, append=n.new_tensor([s["tokens"]]))
    step = src[at]
    img, txt = s["img"].long()[step], s["txt"].long()[step]
    whole = (length == img + txt) & (img > 0)
    skip = torch.where(whole, grid[step].amax(1), 0)
    ends = torch.cumsum(txt + skip, 0)
    base = ends - txt - skip
    head = torch.ones_like(at, dtype=torch.bool)
    head[1:] = seg[at[1:]] != seg[at[:-1]]
    base = base - torch.cummax(torch.where(head, base, 0), 0).values
    k = n - at[run]
    h, w = grid[src, 1], grid[src, 2]
    image = whole[run] & (k < img[run])
    text = base[run] + skip[run] + k - torch.where(whole, img, 0)[run]
    hw = (h * w).clamp(min=1)
    axes = [k // hw, k // w.clamp(min=1) % h.clamp(min=1), k % w.clamp(min=1)]
    return torch.stack([torch.where(image, base[run] + a, text) for a in axes]).to(torch.int32)


def _inverse(s):
    gather = s["gather"].long()
    order = torch.argsort(gather, stable=True)
    off = torch.searchsorted(gather[order], torch.arange(s["traj_tokens"] + 1, device=DEV))
    return off.to(torch.int32), order.to(torch.int32)


def _turn(x, pos, case, sign, dtype):
    """x [tokens, heads, d] rotated by its positions (sign -1: back), in `dtype`."""
    d = case["d"]
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(_sections(d), device=DEV))
    freq = THETA ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d)
    angle = pos.double()[axis].T * freq
    cos, sin = torch.cos(angle).to(dtype)[:, None], (sign * torch.sin(angle)).to(dtype)[:, None]
    x = x.to(dtype)
    a, b = (x[..., 0::2], x[..., 1::2]) if case["interleaved"] else (x[..., :d // 2], x[..., d // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)


def _rope(s):
    at = s["gather"].long()
    q, k = (_turn(s[x][at], s["pos"], s["case"], 1, torch.float32).to(torch.bfloat16) for x in ("q", "k"))
    return q, k, s["v"][at]


def _unrope(s):
    at = s["gather"].long()

    def back(x):
        return x.new_zeros((s["traj_tokens"],) + x.shape[1:]).index_add_(0, at, x).to(torch.bfloat16)

    q, k = (_turn(s[x], s["pos"], s["case"], -1, torch.float32) for x in ("q", "k"))
    return back(q), back(k), back(s["v"].float())


def _attend(s, grads):
    """Blocks of packed rows against the band of keys behind them; a row's sinks beyond the band apart."""
    c, n = s["case"], s["tokens"]
    group, d, sinks = c["hq"] // c["hkv"], c["d"], c["sinks"]
    window, scale = min(c["window"], s["longest"]), 1.0 / math.sqrt(c["d"])
    rows = min(1024, max(128, window))
    blocks = -(-n // rows)
    wide, pad = rows + window - 1, blocks * rows - n
    tok = torch.arange(blocks * rows, device=DEV)
    start = s["cu"].long()[torch.searchsorted(s["cu"].long()[1:], tok.clamp(max=n - 1), right=True)]
    key = tok.view(blocks, rows)[:, :1] - (window - 1) + torch.arange(wide, device=DEV)   # [blocks, wide]
    row = tok.view(blocks, rows, 1)
    hide = (key[:, None] > row) | (key[:, None] <= row - window) | (key[:, None] < start.view(blocks, rows, 1))
    hide = hide.repeat(1, group, 1)                                                       # rows of the group's heads
    first = start[:, None] + torch.arange(sinks, device=DEV)                              # [rows, sinks]
    far = first > tok[:, None] - window
    first = first.clamp(max=n - 1)

    def query(x, g):       # [blocks, group * rows, d]
        x = torch.nn.functional.pad(x[:, g * group:(g + 1) * group].float(), (0, 0, 0, 0, 0, pad))
        return x.view(blocks, rows, group, d).transpose(1, 2).reshape(blocks, group * rows, d)

    def each(x):           # block rows as packed rows [blocks * rows, group, ...]
        return x.view(blocks, group, rows, -1).transpose(1, 2).reshape(blocks * rows, group, -1)

    def block(x):          # and back
        return x.view(blocks, rows, group, -1).transpose(1, 2).reshape(blocks, group * rows, -1)

    def band(x):           # [blocks, wide, d], a view of the padded rows
        x = torch.nn.functional.pad(x, (0, 0, window - 1, pad))
        return x.unfold(0, wide, rows).transpose(1, 2)

    out, lses, dqs, dks, dvs = [], [], [], [], []
    for g in range(c["hkv"]):
        k, v = s["k"][:, g].float(), s["v"][:, g].float()
        q, kb, vb = query(s["q"], g) * scale, band(k), band(v)
        p = torch.bmm(q, kb.transpose(1, 2)).masked_fill_(hide, -math.inf)
        ps = torch.bmm(each(q), k[first].transpose(1, 2)).masked_fill_(far[:, None], -math.inf) if sinks else None
        top = p.amax(2, keepdim=True).clamp_(min=-1e30)
        if sinks:
            top = torch.maximum(top, block(ps.amax(2, keepdim=True)))
            ps = ps.sub_(each(top)).exp_()
        p = p.sub_(top).exp_()
        total = p.sum(2, keepdim=True)
        if sinks:
            total = total + block(ps.sum(2, keepdim=True))
            ps = ps.div_(each(total))
        p = p.div_(total)
        o = torch.bmm(p, vb)
        if sinks:
            o += block(torch.bmm(ps, v[first]))
        out.append(each(o)[:n])
        lses.append(each(top + total.log())[:n, :, 0].T)
        if not grads:
            continue
        do = query(s["do"], g)
        mean = (do * o).sum(2, keepdim=True)
        at = key.clamp(0, n - 1).reshape(-1)
        dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        dv.index_add_(0, at, torch.bmm(p.transpose(1, 2), do).view(-1, d))
        p = torch.bmm(do, vb.transpose(1, 2)).sub_(mean).mul_(p)
        dq = torch.bmm(p, kb)
        dk.index_add_(0, at, torch.bmm(p.transpose(1, 2), q).view(-1, d))
        if sinks:
            at, qr, dor = first.reshape(-1), each(q), each(do)
            dv.index_add_(0, at, torch.bmm(ps.transpose(1, 2), dor).view(-1, d))
            ps = torch.bmm(dor, v[first].transpose(1, 2)).sub_(each(mean)).mul_(ps)
            dq += block(torch.bmm(ps, k[first]))
            dk.index_add_(0, at, torch.bmm(ps.transpose(1, 2), qr).view(-1, d))
        dqs.append(each(dq)[:n] * scale)
        dks.append(dk)
        dvs.append(dv)
    res = dict(o=torch.cat(out, 1).to(torch.bfloat16), lse=torch.cat(lses, 0))
    if grads:
        res.update(dq=torch.cat(dqs, 1).to(torch.bfloat16), dk=torch.stack(dks, 1).to(torch.bfloat16),
                   dv=torch.stack(dvs, 1).to(torch.bfloat16))
    return res


# ------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    if kind == "layout":
        off, tok = _inverse(state)
        return dict(pos=_positions(state), off=off, tok=tok)
    if kind in ("rope", "unrope"):
        q, k, v = _rope(state) if kind == "rope" else _unrope(state)
        return dict(q=q, k=k, v=v)
    return _attend(state, kind == "train")


def _own(kind, s):
    from paper_2607_11185_gb300 import vcs
    c = s["case"]
    if kind == "layout":
        pos = vcs.stream_positions(s["cu"], s["src"], s["img"], s["txt"], s["grid"], check=False)
        off, tok = vcs.gather_inverse(s["gather"], s["traj_tokens"], check=False)
        return dict(pos=pos, off=off, tok=tok)
    if kind in ("rope", "unrope"):
        rope = vcs.rope_plan(c["d"], _sections(c["d"]), THETA, interleaved=c["interleaved"])
        if kind == "rope":
            q, k, v = vcs.gather_rope(s["q"], s["k"], s["v"], s["gather"], s["pos"], rope, check=False)
        else:
            q, k, v = vcs.gather_rope_bwd(s["q"], s["k"], s["v"], s["pos"], *s["inv"], rope, check=False)
        return dict(q=q, k=k, v=v)
    o, lse = vcs.attn_fwd_window(s["q"], s["k"], s["v"], s["cu"], s["longest"], c["window"], c["sinks"], check=False)
    if kind == "fwd":
        return dict(o=o, lse=lse)
    dq, dk, dv = vcs.attn_bwd_window(s["q"], s["k"], s["v"], o, lse, s["do"], s["cu"], s["longest"], c["window"],
                                     c["sinks"], check=False)
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)


def _pairs(c):
    """Visible (query, key) pairs of one head over the layout."""
    length = np.diff(_layout(c)["cu"].astype(np.int64))
    w, s = c["window"], c["sinks"]
    m = np.minimum(length, w)
    seen = m * (m + 1) // 2 + (length - m) * w           # in the window
    beyond = np.maximum(length - w, 0)                   # rows with i >= w see min(sinks, i + 1 - w) more
    t = np.minimum(beyond, s)
    return int((seen + t * (t + 1) // 2 + (beyond - t) * s).sum())


def work(case):
    lay, kind = _layout(case), case["kind"]
    n, t, hq, hkv, d = lay["tokens"], lay["traj_tokens"], case["hq"], case["hkv"], case["d"]
    if kind == "layout":
        return dict(bytes=4 * n + 20 * len(lay["img"]) + 12 * n + 4 * n + 4 * n + 4 * (t + 1), flops=0)
    row = (hq + 2 * hkv) * d * 2
    if kind in ("rope", "unrope"):
        seen = len(np.unique(lay["gather"])) if kind == "rope" else t
        return dict(bytes=(n + seen) * row + 16 * n + (4 * (t + 1) if kind == "unrope" else 0),
                    flops=6 * n * (hq + hkv) * d // 2)
    pairs, rows = _pairs(case) * hq, n * (hq * d * 4 + hkv * d * 4 + hq * 4)
    if kind == "fwd":
        return dict(bytes=rows, flops=4 * d * pairs)
    return dict(bytes=rows + n * (hq * d * 4 + hkv * d * 4), flops=14 * d * pairs)


# ------------------------------------------------------------------ 64 bits

def _exact_positions(lay):
    pos = np.zeros((3, lay["tokens"]), np.int64)
    for b, e in zip(lay["cu"][:-1], lay["cu"][1:]):
        p, i = 0, int(b)
        while i < e:
            s = int(lay["src"][i])
            j = i + int(np.searchsorted(lay["src"][i:e], s, side="right"))
            t, h, w = (int(x) for x in lay["grid"][s])
            if j - i == lay["img"][s] + lay["txt"][s] and lay["img"][s] > 0:
                m = t * h * w
                pos[:, i:i + m] = p + np.indices((t, h, w)).reshape(3, -1)
                i, p = i + m, p + max(t, h, w)
            pos[:, i:j] = p + np.arange(j - i)
            p, i = p + j - i, j
    return pos


def _rotation(lay, case):
    """cos, sin [tokens, 1, d/2] of every pair's angle."""
    angle = np.empty((lay["tokens"], case["d"] // 2))
    axis = np.repeat(np.arange(3), _sections(case["d"]))
    pos = _exact_positions(lay)
    for i, a in enumerate(axis):
        angle[:, i] = pos[a] * THETA ** (-2.0 * i / case["d"])
    angle = torch.from_numpy(angle).to(DEV)
    return torch.cos(angle)[:, None], torch.sin(angle)[:, None]


def _exact_turn(x, cos, sin, case):
    y, h = torch.empty_like(x), case["d"] // 2
    i, j = (slice(0, None, 2), slice(1, None, 2)) if case["interleaved"] else (slice(0, h), slice(h, None))
    y[..., i] = x[..., i] * cos - x[..., j] * sin
    y[..., j] = x[..., j] * cos + x[..., i] * sin
    return y


def _exact_attend(s, lay, grads):
    """Row blocks of one segment and head at a time, every key of the segment before the block's end."""
    c = s["case"]
    group, window, sinks = c["hq"] // c["hkv"], c["window"], c["sinks"]
    scale = c["d"] ** -0.5
    q, k, v = (s[x].double() for x in ("q", "k", "v"))
    o, lse = torch.empty_like(q), torch.empty(c["hq"], s["tokens"], dtype=torch.float64, device=DEV)
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v)) if grads else (None, None, None)
    do = s["do"].double() if grads else None
    step = max(64, min(512, window))
    for b, e in zip(lay["cu"][:-1].tolist(), lay["cu"][1:].tolist()):
        for r in range(b, e, step):
            r1 = min(e, r + step)
            low = max(b, r - window + 1)
            cols = torch.cat([torch.arange(b, min(b + sinks, low), device=DEV), torch.arange(low, r1, device=DEV)])
            i, j = torch.arange(r, r1, device=DEV)[:, None], cols[None]
            seen = (j <= i) & ((i - j < window) | (j - b < sinks))
            for g in range(c["hkv"]):
                h = slice(g * group, (g + 1) * group)
                qh, kk, vv = q[r:r1, h].transpose(0, 1), k[cols, g], v[cols, g]
                x = torch.where(seen, scale * (qh @ kk.T), -math.inf)
                lg = torch.logsumexp(x, 2)
                p = torch.exp(x - lg[..., None])
                oh = p @ vv
                o[r:r1, h], lse[h, r:r1] = oh.transpose(0, 1), lg
                if grads:
                    dh = do[r:r1, h].transpose(0, 1)
                    ds = p * (dh @ vv.T - (dh * oh).sum(2, keepdim=True)) * scale
                    dq[r:r1, h] = (ds @ kk).transpose(0, 1)
                    dk[:, g].index_add_(0, cols, (ds.transpose(1, 2) @ qh).sum(0))
                    dv[:, g].index_add_(0, cols, (p.transpose(1, 2) @ dh).sum(0))
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv) if grads else dict(o=o, lse=lse)


def exact(case, seed):
    kind = case["kind"]
    if kind == "layout":
        return None  # whole numbers
    lay = _layout(case)
    if kind in ("fwd", "train") and work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    if kind in ("fwd", "train"):
        return _exact_attend(s, lay, kind == "train")
    at = torch.from_numpy(lay["gather"].astype(np.int64)).to(DEV)
    cos, sin = _rotation(lay, case)
    if kind == "rope":
        return dict(q=_exact_turn(s["q"].double()[at], cos, sin, case), k=_exact_turn(s["k"].double()[at], cos, sin, case),
                    v=s["v"].double()[at])

    def back(x):
        return x.new_zeros((s["traj_tokens"],) + x.shape[1:]).index_add_(0, at, x)

    return dict(q=back(_exact_turn(s["q"].double(), cos, -sin, case)),
                k=back(_exact_turn(s["k"].double(), cos, -sin, case)), v=back(s["v"].double()))
