"""Linear attention with a decay for each head, and distillation from a teacher's top logits, as timed cases.

A policy whose history runs through linear attention keeps one state a key/value head, S_t = e^g S_{t-1} + k_t v_t^T,
from which the head's queries read o_t = scale q_t S_t.  It is trained over the segments of its trajectories, from
the top logits that a teacher left for every trained token, and answers token by token.  Each case is one of these:

  fwd      the outputs of a layout's segments (scoring, reference policy)
  prompt   the same from a state that each sequence has and to the one it goes on with (serving)
  train    outputs and the gradients of q, k and v
  step     one token of each sequence, its state updated in place
  kl       the divergence of every row from its teacher, and their weighted sum (evaluation)
  distill  the same with the gradient of the logits

Where `own` is false they are computed by elementary torch operations in 32 bits, chunk by chunk with the
states between the chunks (their sums over rows in 64).  The lengths that fix a case's shapes come from its own
`shape` number, the tensors from the seed.
"""
import functools
import math

import numpy as np
import torch

own = False
DEV = "cuda"
CHUNK = 128


def _seq(name, kind, heads, seqs, length, cut=0, keep=0, steps=(1, 1), txt=(0, 0), still=False, shape=1):
    """`seqs` sequences of length[0] .. length[1] tokens; with a cut, trajectories of steps[0] .. steps[1] screenshots
    of that many tokens and responses of txt[0] .. txt[1], cut into segments.  still: head 0 does not decay."""
    return dict(name=name, kind=kind, hq=heads[0], hkv=heads[1], d=heads[2], seqs=seqs, len_lo=length[0],
                len_hi=length[1], cut=cut, keep=keep, steps_lo=steps[0], steps_hi=steps[1], txt_lo=txt[0],
                txt_hi=txt[1], still=still, shape=shape)


def _rows(name, kind, rows, vocab, top, fp32=False, temperature=1.0, pad=0, mapped=False, absent=0.0, idle=0.0):
    """`rows` rows of `vocab` logits in a buffer of vocab + pad columns, `top` teacher entries each.  mapped: the lists
    are the trajectory's, read by row; absent: share of entries left out; idle: share of rows of weight 0."""
    return dict(name=name, kind=kind, rows=rows, vocab=vocab, top=top, fp32=fp32, temperature=temperature, pad=pad,
                mapped=mapped, absent=absent, idle=idle)


LONG = dict(cut=8, steps=(50, 50), txt=(512, 512))      # long-horizon rollouts of 2,700-token screenshots
SHORT = dict(cut=3, steps=(5, 15), txt=(64, 256))       # short rollouts of 1,024-token screenshots


def listed():
    return [
        # the next token of one sequence: latency
        _seq("step_one", "step", (28, 4, 128), 1, (1, 1)),
        # the next token of a full batch of rollouts (268 MB of states)
        _seq("step_batch", "step", (40, 8, 128), 512, (1, 1)),
        # a few short observations appended to running sequences: latency
        _seq("prompt_short", "prompt", (14, 2, 64), 3, (1, 300)),
        # two long prompts of odd lengths, a key/value head for each query head
        _seq("prompt_long", "prompt", (16, 16, 128), 2, (30001, 40001), still=True),
        # scoring of one four-step rollout of 256-token screenshots: latency
        _seq("fwd_tiny", "fwd", (2, 1, 64), 1, (256, 256), cut=2, steps=(4, 4), txt=(32, 32)),
        # scoring of one long rollout: seven segments of 25,696 to 46,176 tokens at the largest row size
        _seq("fwd_long", "fwd", (40, 8, 128), 1, (2700, 2700), **LONG),
        # the update of a batch of short rollouts with 64-wide heads
        _seq("train_d64", "train", (14, 2, 64), 8, (1024, 1024), **SHORT, still=True, shape=2),
        # the update of one long rollout
        _seq("train_long", "train", (40, 8, 128), 1, (2700, 2700), **LONG),
        # the divergence at one token: latency
        _rows("kl_one", "kl", 1, 32000, 20),
        # evaluation of a batch of responses against lists stored by trajectory token, some shorter than others, an odd
        # vocabulary in 32 bits
        _rows("kl_fp32", "kl", 512, 99991, 100, fp32=True, temperature=2.0, mapped=True, absent=0.2),
        # the update on short responses, a padded vocabulary, rows of which some are not trained
        _rows("distill_short", "distill", 600, 32000, 32, pad=768, absent=0.1, idle=0.25),
        # the update on a batch of long responses at a large vocabulary
        _rows("distill_long", "distill", 4096, 131072, 64, temperature=1.5, mapped=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["step", "prompt", "fwd", "train", "train", "kl", "distill", "distill"])
    if kind in ("kl", "distill"):
        vocab = log(500, 160_000)
        fp32 = rng.random() < 0.4
        rows = log(1, max(2, min(20_000, 5e8 / vocab / (2 if fp32 else 1))))
        return _rows(None, kind, rows, vocab, log(1, min(256, vocab)), fp32, rng.choice([0.5, 1.0, 1.0, 2.0, 3.7]),
                     rng.choice([0, 0, 1, 8, 61, 128]), rng.random() < 0.5, rng.choice([0.0, 0.0, 0.1, 0.5]),
                     rng.choice([0.0, 0.0, 0.3]))
    heads = rng.choice([(1, 1, 64), (2, 1, 64), (6, 6, 64), (14, 2, 64), (6, 2, 128), (16, 16, 128), (28, 4, 128),
                        (40, 8, 128)])
    shape, still = rng.randrange(1, 1 << 20), rng.random() < 0.3
    if kind == "step":
        return _seq(None, kind, heads, log(1, min(4096, 2e8 / (heads[1] * heads[2] ** 2 * 4))), (1, 1), still=still,
                    shape=shape)
    most = min(400_000, int((2.4e9 if kind == "fwd" else 1.2e9) / ((heads[0] + heads[1]) * heads[2])))
    tokens = log(2, most)
    if kind == "prompt" or rng.random() < 0.3:
        seqs = log(1, min(64, tokens))
        return _seq(None, kind, heads, seqs, (0, max(1, 2 * tokens // seqs)), still=still, shape=shape)
    img, txt, steps, cut, keep = log(16, 2700), log(4, 512), rng.randrange(1, 30), rng.randrange(1, 9), rng.randrange(3)
    each = steps * (img * (1 + keep / cut) + txt * (1 + steps / 2 / cut))
    if each > most:
        img, txt, steps, each = 64, 16, 3, 240 * (1 + keep / cut)
    return _seq(None, kind, heads, max(1, int(tokens / each)), (max(1, img // 2), img), cut, keep,
                (max(1, steps // 2), steps), (txt // 2, txt), still, shape)


# ------------------------------------------------------------------ inputs

def _lengths(c):
    return _lengths_of(*(c[k] for k in ("shape", "seqs", "len_lo", "len_hi", "cut", "keep", "steps_lo", "steps_hi",
                                        "txt_lo", "txt_hi")))


@functools.lru_cache(maxsize=8)
def _lengths_of(shape, seqs, l0, l1, cut, keep, s0, s1, t0, t1):
    """Tokens of each sequence, or of each segment of the trajectories."""
    rng = np.random.default_rng(shape)
    if not cut:
        out = rng.integers(l0, l1, size=seqs, endpoint=True)
        out[0] += not out.any()
        return out
    out = []
    for n in rng.integers(s0, s1, size=seqs, endpoint=True):
        img, txt = rng.integers(l0, l1, size=n, endpoint=True), rng.integers(t0, t1, size=n, endpoint=True)
        done, stop = 0, min(int(n), keep + cut)
        while True:
            out.append(int(txt[:stop].sum() + img[max(0, done - keep):stop].sum()))
            if stop == n:
                break
            done, stop = stop, min(int(n), stop + cut)
    return np.array(out)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _decays(c):
    """Head h forgets at the rate 2^(-8 (h + 1) / heads) a token."""
    g = -(2.0 ** (-8.0 * torch.arange(1, c["hkv"] + 1, dtype=torch.float32, device=DEV) / c["hkv"]))
    if c["still"]:
        g[0] = 0.0
    return g


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if case["kind"] in ("kl", "distill"):
        return _prepare_rows(case, gen)
    kind, hq, hkv, d = (case[k] for k in ("kind", "hq", "hkv", "d"))
    lens = _lengths(case)
    n = int(lens.sum())
    s = dict(case=case, tokens=n, decay=_decays(case))
    s["cu"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(DEV)
    s["q"], s["k"], s["v"] = _normal(gen, n, hq, d), _normal(gen, n, hkv, d), _normal(gen, n, hkv, d)
    if kind == "train":
        s["do"] = _normal(gen, n, hq, d)
    if kind in ("prompt", "step"):  # states of running sequences
        s["state"] = torch.randn(len(lens), hkv, d, d, generator=gen, device=DEV)
    return s


def _prepare_rows(c, gen):
    rows, vocab, top = c["rows"], c["vocab"], c["top"]
    lists = rows + rows // 3 if c["mapped"] else rows

    def rand(*shape):
        return torch.rand(shape, generator=gen, device=DEV)

    # entries spread over the vocabulary, each in a range of its own, in any order; the best one 5 to 15 above the rest
    at = torch.arange(top, device=DEV)
    ids = (at * vocab // top + (rand(lists, top) * (vocab // top)).long().clamp(max=vocab // top - 1))
    ids = ids.gather(1, torch.argsort(rand(lists, top), dim=1))
    logits = 8.0 + 3.0 * torch.randn(lists, top, generator=gen, device=DEV) - 0.1 * at
    student = torch.empty(rows, vocab + c["pad"], device=DEV, dtype=torch.float32 if c["fp32"] else torch.bfloat16)
    student.normal_(generator=gen).mul_(2.0)
    s = dict(case=c, rows=None)
    mine = torch.arange(rows, device=DEV)
    if c["mapped"]:
        mine = torch.randperm(lists, generator=gen, device=DEV)[:rows]
        s["rows"] = mine.to(torch.int32)
    near = logits[mine] + torch.randn(rows, top, generator=gen, device=DEV)   # a student on its way to the teacher
    student.scatter_(1, ids[mine], near.to(student.dtype))
    ids = torch.where(rand(lists, top) < c["absent"], -1, ids)
    weights = (0.5 + rand(rows)) / rows
    s["weights"] = torch.where(rand(rows) < c["idle"], torch.zeros_like(weights), weights)
    s["ids"], s["logits"], s["student"] = ids.to(torch.int32), logits, student[:, :vocab]
    return s


# ------------------------------------------------------------------ plain forms

def _chunks(cu):
    """Token of every place of every chunk, whether it is one, and each segment's chunks."""
    length = torch.diff(cu)
    count = (length + CHUNK - 1) // CHUNK
    seg = torch.repeat_interleave(torch.arange(len(length), device=DEV), count)
    first = torch.cumsum(count, 0) - count
    off = (torch.arange(len(seg), device=DEV) - first[seg]) * CHUNK
    tok = off[:, None] + torch.arange(CHUNK, device=DEV)
    real = tok < length[seg][:, None]
    return torch.where(real, tok + cu[:-1][seg][:, None], 0), real, first, count, (length[seg] - off).clamp(max=CHUNK)


def _attend(q, k, v, decay, cu, scale, state=None, behind=False):
    """Linear attention over packed tokens; behind: a token sees the ones from itself on (the sums of a key's
    gradient).  Where the keys have more heads than the queries, a query head reads its whole group.  Returns the
    outputs in 32 bits and the states behind the segments."""
    tok, real, first, count, size = _chunks(cu)
    heads = min(q.shape[1], k.shape[1])
    gq, gk = q.shape[1] // heads, k.shape[1] // heads
    d, n = q.shape[2], tok.shape[0]
    at = torch.arange(CHUNK, device=DEV)
    if behind:                                             # time runs the other way in every chunk
        at, since = (size[:, None] - 1 - at).clamp(min=0), at[None].expand(n, -1)
    else:
        since = (size[:, None] - 1 - at).clamp(min=0)      # tokens from a key to the chunk's end
        at = at[None].expand(n, -1)                        # tokens from the chunk's beginning to a query
    own_state = torch.zeros(n, heads, d, d, device=DEV)

    def part(x, h, g):                                     # [chunks, g * CHUNK, d] of the head's group
        x = x[:, h * g:(h + 1) * g].float()[tok] * real[:, :, None, None]
        return x.transpose(1, 2).reshape(n, g * CHUNK, d)

    for h in range(heads):
        w = torch.exp(decay[h] * since).repeat(1, gk)[..., None]
        own_state[:, h] = torch.bmm((part(k, h, gk) * w).transpose(1, 2), part(v, h, gk))
    before = torch.empty_like(own_state)                   # the state that each chunk starts from
    now = torch.zeros(len(count), heads, d, d, device=DEV) if state is None else state.clone()
    most = int(count.max()) if len(count) else 0
    order = torch.argsort(count, descending=True, stable=True)
    alive = (count[order][None] > torch.arange(most, device=DEV)[:, None]).sum(1).tolist()
    for i in range(most):
        seg = order[:alive[i]]
        c = first[seg] + (count[seg] - 1 - i if behind else i)
        cur = now[seg]
        before[c] = cur
        now[seg] = cur * torch.exp(decay * size[c][:, None])[..., None, None] + own_state[c]
    gap = torch.arange(CHUNK, device=DEV)
    gap = gap[:, None] - gap[None]
    gap = -gap if behind else gap
    out = torch.empty(q.shape, device=DEV)
    for h in range(heads):
        fade = torch.where(gap >= 0, torch.exp(decay[h] * gap.clamp(min=0)), 0.0).repeat(gq, gk)
        qh, kh, vh = part(q, h, gq), part(k, h, gk), part(v, h, gk)
        o = torch.bmm(torch.bmm(qh, kh.transpose(1, 2)).mul_(fade), vh)
        o += torch.bmm(qh, before[:, h]) * torch.exp(decay[h] * (at + 1)).repeat(1, gq)[..., None]
        o = o.view(n, gq, CHUNK, d).transpose(1, 2)
        out[:, h * gq:(h + 1) * gq].index_put_((tok[real],), o[real] * scale)
    return out, now


def _plain(s):
    c, cu = s["case"], s["cu"].long()
    q, k, v, g = s["q"], s["k"], s["v"], s["decay"]
    scale = c["d"] ** -0.5
    if c["kind"] == "step":
        state = s["state"].mul_(torch.exp(g)[:, None, None]).add_(k.float()[..., None] * v.float()[..., None, :])
        qg = q.float().view(-1, c["hkv"], c["hq"] // c["hkv"], c["d"])
        return dict(o=(torch.matmul(qg, state) * scale).view(q.shape).to(q.dtype), state=state)
    o, state = _attend(q, k, v, g, cu, scale, s.get("state"))
    res = dict(o=o.to(q.dtype))
    if c["kind"] == "prompt":
        res["state"] = state
    if c["kind"] == "train":
        do = s["do"]
        res["dq"] = _attend(do, v, k, g, cu, scale)[0].to(q.dtype)
        res["dk"] = _attend(v, do, q, g, cu, scale, behind=True)[0].to(k.dtype)
        res["dv"] = _attend(k, q, do, g, cu, scale, behind=True)[0].to(v.dtype)
    return res


def _plain_rows(s):
    c, w = s["case"], s["weights"]
    ids, t = (s["ids"], s["logits"]) if s["rows"] is None else (s["ids"][s["rows"].long()], s["logits"][s["rows"].long()])
    here = ids >= 0
    t = (t / c["temperature"]).masked_fill(~here, -math.inf)
    some = here.any(1) & (w != 0)
    p = torch.exp(t - t.amax(1, keepdim=True).clamp(min=-1e30))
    total = p.sum(1, keepdim=True).clamp(min=1e-30)
    p = torch.where(some[:, None], p / total, 0.0)
    z = s["student"].float() / c["temperature"]
    top = z.amax(1, keepdim=True)
    q = torch.exp(z - top)
    norm = q.sum(1, keepdim=True, dtype=torch.float64)
    at = ids.long().clamp(min=0)
    logq = z.gather(1, at).double() - top.double() - torch.log(norm)
    kl = torch.where(p > 0, p.double() * (torch.log(p.double().clamp(min=1e-300)) - logq), 0.0).sum(1)
    res = dict(loss=(w.double() * kl).sum().float().view(1), kl=kl.float())
    if c["kind"] == "distill":
        q = q.mul_((1.0 / norm).float() * some[:, None]).scatter_add_(1, at, -p)
        res["dlogits"] = q.mul_(w[:, None] / c["temperature"]).to(s["student"].dtype)
    return res


# ------------------------------------------------------------------ one pass

def run(state):
    rows = state["case"]["kind"] in ("kl", "distill")
    if own:
        return _own_rows(state) if rows else _own(state)
    return _plain_rows(state) if rows else _plain(state)


def _own(s):
    from paper_2607_11185_gb300 import vcs
    kind = s["case"]["kind"]
    if kind == "step":
        o = vcs.linear_attn_step(s["q"], s["k"], s["v"], s["decay"], s["state"], check=False)
        return dict(o=o, state=s["state"])
    if kind == "prompt":
        o, state = vcs.linear_attn_fwd(s["q"], s["k"], s["v"], s["decay"], s["cu"], state=s["state"], with_state=True,
                                       check=False)
        return dict(o=o, state=state)
    o, _ = vcs.linear_attn_fwd(s["q"], s["k"], s["v"], s["decay"], s["cu"], check=False)
    if kind == "fwd":
        return dict(o=o)
    dq, dk, dv = vcs.linear_attn_bwd(s["q"], s["k"], s["v"], s["do"], s["decay"], s["cu"], check=False)
    return dict(o=o, dq=dq, dk=dk, dv=dv)


def _own_rows(s):
    from paper_2607_11185_gb300 import vcs
    grad = s["case"]["kind"] == "distill"
    loss, kl, dlogits = vcs.distill_topk(s["student"], s["ids"], s["logits"], s["weights"], teacher_rows=s["rows"],
                                         temperature=s["case"]["temperature"], with_grad=grad, check=False)
    return dict(loss=loss, kl=kl, dlogits=dlogits) if grad else dict(loss=loss, kl=kl)


def work(case):
    kind = case["kind"]
    if kind in ("kl", "distill"):
        busy = case["rows"] * (1 - case["idle"])
        size = case["vocab"] * (4 if case["fp32"] else 2)
        moved = busy * size + (case["rows"] * size if kind == "distill" else 0)
        return dict(bytes=int(moved + case["rows"] * (8 * case["top"] + 12)),
                    flops=int(busy * case["vocab"] * (6 if kind == "distill" else 3)))
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens = _lengths(case)
    n = int(lens.sum())
    moved, states = 2 * n * d * (2 * hq + 2 * hkv), len(lens) * hkv * d * d * 4
    if kind in ("prompt", "step"):
        moved += 2 * states
    if kind == "train":
        moved *= 2
    # a product with the state for each query head's row, an update for each key/value head's; the gradients' are
    # dq, dk and dv from the states and the two states' updates
    flops = 2 * n * d * d * (hq + hkv) + (2 * n * d * d * (2 * hq + 3 * hkv) if kind == "train" else 0)
    return dict(bytes=moved, flops=flops)


# ------------------------------------------------------------------ 64 bits

def _walk(lens, cu, names, tensors, step, back):
    """Calls step(active segments, tokens' rows...) for every position of the segments, longest first, and packs what it
    returns; positions in order or from the last one back."""
    order = np.argsort(-lens, kind="stable")
    longest, block = int(lens.max(initial=0)), 256
    start, size = cu[:-1][order], lens[order]
    outs = {}
    blocks = list(range(0, longest, block))
    for b in reversed(blocks) if back else blocks:
        act = int((size > b).sum())
        at = b + np.arange(block)
        ok = at[None] < size[:act, None]
        idx = torch.from_numpy(np.where(ok, start[:act, None] + at[None], 0)).to(DEV)
        rows = [x[idx].double() for x in tensors]
        res = {}
        times = range(min(block, longest - b))
        for t in reversed(times) if back else times:
            a = int((size > b + t).sum())
            for name, y in zip(names, step(a, *(x[:a, t] for x in rows))):
                if name not in res:
                    res[name] = y.new_zeros(act, block, *y.shape[1:])
                res[name][:a, t] = y
        okt = torch.from_numpy(ok).to(DEV)
        for name, y in res.items():
            if name not in outs:
                outs[name] = y.new_zeros(int(lens.sum()), *y.shape[2:])
            outs[name][idx[okt]] = y[okt]
    return outs, torch.from_numpy(order).to(DEV)


def _exact_seq(case, s):
    """Token by token, by the recurrence."""
    hq, hkv, d, kind = (case[k] for k in ("hq", "hkv", "d", "kind"))
    lens = _lengths(case)
    cu = np.concatenate([[0], np.cumsum(lens)])
    lam, scale = torch.exp(s["decay"].double())[:, None, None], d ** -0.5
    order = torch.from_numpy(np.argsort(-lens, kind="stable")).to(DEV)
    mem = s["state"].double()[order] if "state" in s else torch.zeros(len(lens), hkv, d, d, dtype=torch.float64, device=DEV)

    def forth(a, q, k, v, *do):
        m = mem[:a].mul_(lam).addcmul_(k[..., None], v[..., None, :])
        res = [torch.matmul(q.view(a, hkv, -1, d), m).view(a, hq, d) * scale]
        if do:
            res.append(torch.matmul(do[0].reshape(a, hkv, -1, d), m.transpose(2, 3)).view(a, hq, d) * scale)
        return res

    train = kind == "train"
    given = [s["q"], s["k"], s["v"]] + ([s["do"]] if train else [])
    res, _ = _walk(lens, cu, ["o", "dq"], given, forth, False)
    if kind in ("prompt", "step"):
        state = torch.empty_like(mem)
        state[order] = mem
        res["state"] = state
    if train:
        rem = torch.zeros_like(mem)

        def back(a, q, k, v, do):
            m = rem[:a].mul_(lam)
            m += torch.matmul(q.reshape(a, hkv, -1, d).transpose(2, 3), do.reshape(a, hkv, -1, d))
            return (torch.matmul(m, v[..., None])[..., 0] * scale, torch.matmul(k[..., None, :], m)[..., 0, :] * scale)

        res.update(_walk(lens, cu, ["dk", "dv"], given, back, True)[0])
    for name, like in (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v")):   # no tokens at all
        if (train or name == "o") and name not in res:
            res[name] = s[like].double()
    return res


def _exact_rows(case, s):
    temp = float(case["temperature"])
    lists = (lambda x: x) if s["rows"] is None else (lambda x: x[s["rows"].long()])
    ids, t, w = lists(s["ids"]).long(), lists(s["logits"]).double() / temp, s["weights"].double()
    kl = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    grad = torch.zeros(case["rows"], case["vocab"], device=DEV, dtype=torch.float64) if case["kind"] == "distill" else None
    step = max(1, int(2e8 / case["vocab"]))
    for r in range(0, case["rows"], step):
        at = slice(r, r + step)
        logq = torch.log_softmax(s["student"][at].double() / temp, 1)
        real = ids[at] >= 0
        logp = torch.log_softmax(torch.where(real, t[at], -math.inf), 1)
        use = real & (w[at] != 0)[:, None]
        p = torch.where(use, torch.exp(logp), 0.0)
        col = ids[at].clamp(min=0)
        kl[at] = torch.where(use, p * (logp - logq.gather(1, col)), 0.0).sum(1)
        if grad is not None:
            dense = torch.zeros_like(logq).scatter_add_(1, col, p)
            grad[at] = (torch.exp(logq) * p.sum(1, keepdim=True) - dense) * (w[at] / temp)[:, None]
    res = dict(loss=(w * kl).sum().view(1), kl=kl)
    if grad is not None:
        res["dlogits"] = grad
    return res


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rows(case, s) if case["kind"] in ("kl", "distill") else _exact_seq(case, s)
