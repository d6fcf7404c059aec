"""Linear attention and distillation on the host (CPU only): refusals and workspaces."""
import numpy as np
import pytest
import torch

A, BIG = 1 << 20, 1 << 40


@pytest.fixture(scope="module")
def vcs():
    from paper_2607_11185_gb300 import vcs as v
    return v


def far(i):
    """Addresses too far apart for the buffers to overlap."""
    return (i + 1) << 44


def fwd(vcs, **kw):
    x = dict(q=far(0), k=far(1), v=far(2), g=far(3), cu=far(4), ns=1, nt=10, hq=2, hkv=1, d=64, sc=0.0, si=None, so=None,
             o=far(5), ws=A, n=BIG) | kw
    return vcs.vcs_linear_attn_fwd(*(x[i] for i in ("q", "k", "v", "g", "cu", "ns", "nt", "hq", "hkv", "d", "sc", "si",
                                                    "so", "o", "ws", "n")), 0)


def bwd(vcs, **kw):
    x = dict(q=far(0), k=far(1), v=far(2), do=far(6), g=far(3), cu=far(4), ns=1, nt=10, hq=2, hkv=1, d=64, sc=0.0,
             dq=far(5), dk=far(7), dv=far(8), ws=A, n=BIG) | kw
    return vcs.vcs_linear_attn_bwd(*(x[i] for i in ("q", "k", "v", "do", "g", "cu", "ns", "nt", "hq", "hkv", "d", "sc",
                                                    "dq", "dk", "dv", "ws", "n")), 0)


def step(vcs, **kw):
    x = dict(q=far(0), k=far(1), v=far(2), g=far(3), nt=10, hq=2, hkv=1, d=64, sc=0.0, so=far(4), o=far(5), w=None) | kw
    return vcs.vcs_linear_attn_step(*(x[i] for i in ("q", "k", "v", "g", "nt", "hq", "hkv", "d", "sc", "so", "o", "w")), 0)


def test_linear_refusals(vcs):
    for f in (fwd, bwd, step):
        for kw in (dict(q=None), dict(k=None), dict(v=None), dict(g=None), dict(nt=-1), dict(hq=0), dict(hkv=-1),
                   dict(q=far(0) + 8), dict(k=far(1) + 2)):
            assert f(vcs, **kw) == 1, kw
        for kw in (dict(d=96), dict(d=256), dict(hq=3, hkv=2), dict(hq=1, hkv=2), dict(hq=65536)):
            assert f(vcs, **kw) == 2, kw
        assert f(vcs, nt=1 << 31) == 4 and f(vcs, nt=(1 << 31) - 256) == 4
    for f in (fwd, bwd):
        for kw in (dict(cu=None), dict(ns=-1)):
            assert f(vcs, **kw) == 1, kw
        for kw in (dict(ws=None), dict(ws=A + 16), dict(n=255)):
            assert f(vcs, **kw) == 8, kw
    row = 10 * 2 * 64 * 2
    for kw in (dict(o=None), dict(o=far(5) + 8), dict(o=far(0)), dict(o=far(0) + row - 16), dict(o=far(0) - row + 16),
               dict(o=far(1)), dict(o=far(2)), dict(si=far(9) + 4), dict(so=far(9) + 4), dict(si=far(9), so=far(9)),
               dict(so=far(5))):
        assert fwd(vcs, **kw) == 1, kw
    for kw in (dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dv=far(8) + 8), dict(dv=far(7)),
               dict(dq=far(6)), dict(dk=far(0)), dict(dv=far(7) + 64)):
        assert bwd(vcs, **kw) == 1, kw
    for kw in (dict(so=None), dict(so=far(4) + 4), dict(o=None), dict(o=far(0)), dict(so=far(2)), dict(o=far(4) + 64)):
        assert step(vcs, **kw) == 1, kw


def test_linear_workspaces(vcs):
    for size, call in ((vcs.vcs_linear_attn_fwd_workspace_size, fwd), (vcs.vcs_linear_attn_bwd_workspace_size, bwd)):
        last = 0
        for nt in (0, 1, 128, 5000, 50_000, 1_000_000):
            n = size(3, nt, 8, 2, 128)
            assert n >= max(256, last) and n % 256 == 0
            last = n
            assert call(vcs, ns=3, nt=nt, hq=8, hkv=2, d=128, n=n - 1) == 8
        for bad in ((-1, 5, 2, 1, 64), (1, -5, 2, 1, 64), (1, 5, 0, 1, 64), (1, 5, 2, 0, 64), (1, 5, 2, 1, 0)):
            assert size(*bad) == 0


def distill(vcs, **kw):
    x = dict(z=far(0), t=0, rows=4, vocab=100, ld=100, ids=far(1), tl=far(2), top=8, lists=4, map=None, w=far(3), temp=1.0,
             loss=far(4), kl=far(5), g=far(6), ldg=100, ws=A, n=BIG) | kw
    return vcs.vcs_distill_topk(*(x[i] for i in ("z", "t", "rows", "vocab", "ld", "ids", "tl", "top", "lists", "map", "w",
                                                 "temp", "loss", "kl", "g", "ldg", "ws", "n")), 0)


def test_distill_refusals(vcs):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(z=None), dict(ids=None), dict(tl=None), dict(w=None), dict(loss=None), dict(kl=None), dict(rows=-1),
               dict(vocab=0), dict(vocab=-4), dict(top=0), dict(lists=-1), dict(lists=3), dict(ld=99), dict(ldg=99),
               dict(temp=0.0), dict(temp=-1.0), dict(temp=nan), dict(temp=inf), dict(z=far(0) + 1), dict(g=far(6) + 1),
               dict(t=1, z=far(0) + 2), dict(t=1, g=far(6) + 2), dict(ids=far(1) + 2), dict(tl=far(2) + 1),
               dict(w=far(3) + 2), dict(loss=far(4) + 2), dict(kl=far(5) + 2), dict(map=far(7) + 2),
               dict(g=far(0), ldg=101), dict(g=far(0) + 2), dict(g=far(0) - 798), dict(g=far(1)), dict(g=far(3)),
               dict(kl=far(0)), dict(loss=far(3) + 4), dict(kl=far(4)), dict(kl=far(6) + 4), dict(loss=far(2))):
        assert distill(vcs, **kw) == 1, kw
    for kw in (dict(t=2), dict(t=-1), dict(top=1025)):
        assert distill(vcs, **kw) == 2, kw
    for kw in (dict(rows=1 << 31, lists=1 << 31), dict(lists=1 << 31), dict(vocab=1 << 31, ld=1 << 31, ldg=1 << 31),
               dict(ld=1 << 62), dict(ldg=1 << 62)):
        assert distill(vcs, **kw) == 4, kw
    for kw in (dict(ws=None), dict(ws=A + 16), dict(n=vcs.vcs_distill_topk_workspace_size(4) - 1)):
        assert distill(vcs, **kw) == 8, kw
    assert vcs.vcs_distill_topk_workspace_size(-5) == vcs.vcs_distill_topk_workspace_size(0) >= 256


def test_tensors_on_the_host_are_refused(vcs):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    for f in (lambda: vcs.linear_attn_fwd(x, x, x, torch.zeros(2), cu),
              lambda: vcs.linear_attn_bwd(x, x, x, x, torch.zeros(2), cu),
              lambda: vcs.linear_attn_step(x, x, x, torch.zeros(2), torch.zeros(4, 2, 64, 64)),
              lambda: vcs.distill_topk(torch.zeros(4, 9), cu.view(1, 2), torch.zeros(1, 2), torch.zeros(4)),
              lambda: vcs.distill_topk(torch.zeros(4, 9).half(), cu.view(1, 2), torch.zeros(1, 2), torch.zeros(4))):
        with pytest.raises(ValueError):
            f()


# ------------------------------------------------------------------ how the forward's and backward's work is divided
CHUNK, GRID, WHOLE = 128, 152, 16


def pieces(lens, heads, bound):
    """The documented rule, CTA by CTA: lists of (segment, head, c0, c1) and whether sequences are cut."""
    nch = [-(-n // CHUNK) for n in lens]
    off = np.concatenate([[0], np.cumsum(nch)])
    total, cut = int(off[-1]) * heads, max(nch, default=0) > WHOLE
    grid = min(GRID, bound)
    size = -(-total // grid) if grid else 0
    out = []
    for b in range(grid):
        g, hi, mine = min(size * b, total), min(size * (b + 1), total), []
        while g < hi:
            seg = int(np.searchsorted(off, g // heads, side="right")) - 1
            head = (g - int(off[seg]) * heads) // nch[seg]
            base = int(off[seg]) * heads + head * nch[seg]
            if not cut and g != base:
                g = base + nch[seg]
                continue
            c0, c1 = g - base, min(nch[seg], hi - base) if cut else nch[seg]
            mine.append((seg, head, c0, c1))
            g = base + c1
        out.append(mine)
    return out, cut


def test_every_chunk_is_taken_once_and_cuts_lead_to_the_next_cta():
    rng = np.random.default_rng(0)
    for _ in range(120):
        heads = int(rng.integers(1, 9))
        most = int(rng.choice([5, 300, 3000, 60_000]))
        lens = [int(x) for x in rng.integers(0, most, size=int(rng.integers(1, 40)))]
        if rng.random() < 0.2:
            lens[0] = int(rng.integers(1, 400_000))
        work, cut = pieces(lens, heads, heads * (sum(lens) // CHUNK + len(lens)))
        seen = {}
        for b, mine in enumerate(work):
            for i, (seg, head, c0, c1) in enumerate(mine):
                assert c1 > c0
                assert c0 == 0 or (cut and i == 0)                      # only the first goes on from another CTA
                assert c1 == -(-lens[seg] // CHUNK) or (cut and i == len(mine) - 1)
                at, last = seen.get((seg, head), (0, None))
                assert c0 == at and (last is None or last == b - 1)     # cuts lead to the very next CTA
                seen[seg, head] = c1, b
        assert {k: v[0] for k, v in seen.items()} == {(s, h): -(-n // CHUNK) for s, n in enumerate(lens) if n
                                                      for h in range(heads)}
        if not cut:  # no CTA takes more than its share and one sequence
            share = -(-sum(c1 - c0 for m in work for *_, c0, c1 in m) // max(len(work), 1))
            assert max((sum(c1 - c0 for *_, c0, c1 in m) for m in work), default=0) <= share + WHOLE


def parts_of(lens, heads, decays, back):
    """The documented rule for the states at the cuts: (cuts, parts, size); a cut (t, sequence, chunk e in it, chunks of
    its own that it needs), its parts' (cut, first chunk, end), the nearest first."""
    nch = [-(-n // CHUNK) for n in lens]
    work, cut = pieces(lens, heads, heads * (sum(lens) // CHUNK + len(lens)))
    keep = [int(min(150 / max(-g * 1.4426950408889634 * CHUNK, 1e-30), 2.0 ** 30)) + 2 for g in decays]
    cuts = []
    for t, mine in enumerate(work):
        if cut and mine and mine[-1][3] < nch[mine[-1][0]]:
            seg, head, c0, e = mine[-1]
            nxt = work[t + 1][0]
            cuts.append((t, (seg, head), e, min(keep[head], nxt[3] - nxt[2] if back else e - c0)))
    need = np.array([c[3] for c in cuts] or [0])
    sizes = []
    for waves in (1, 2, 3):
        s = 4
        while (-(-need // s)).sum() > waves * len(work):
            s += 1
        sizes.append(s)
    size = min(sizes, key=lambda s: (sizes.index(s) + 1) * (s + 3))
    parts = []
    for t, _, e, n in cuts:
        for j in range(-(-n // size)):
            near, away = j * size, min((j + 1) * size, n)
            parts.append((t, e + near, e + away) if back else (t, e - away, e - near))
    assert len(parts) <= 3 * len(work)
    return cuts, parts, size


@pytest.mark.parametrize("back", [False, True])
def test_the_parts_hold_what_every_cut_needs_once(back):
    rng = np.random.default_rng(1)
    for _ in range(60):
        heads = int(rng.integers(1, 9))
        lens = [int(x) for x in rng.integers(0, int(rng.choice([300, 3000, 40_000])), size=int(rng.integers(1, 20)))]
        lens[0] = int(rng.integers(2100, 200_000))
        decays = [-float(10 ** rng.uniform(-6, 1)) if rng.random() < 0.8 else 0.0 for _ in range(heads)]
        cuts, parts, size = parts_of(lens, heads, decays, back)
        assert cuts
        by = {t: [(a, b) for u, a, b in parts if u == t] for t, *_ in cuts}
        for t, (seg, head), e, _ in cuts:
            nch = -(-lens[seg] // CHUNK)
            want, at, faded = (nch if back else 0), e, False
            for u, seq, eu, n in (cuts if back else cuts[::-1]):
                if seq != (seg, head) or (u < t if back else u > t) or faded:
                    continue
                for a, b in by[u]:
                    near = a - e if back else e - b
                    assert near == abs(at - e)                          # the next chunks, nothing twice
                    if -decays[head] * 1.4426950408889634 * CHUNK * near > 150:
                        faded = True
                        break
                    at = b if back else a
                faded = faded or -decays[head] * 1.4426950408889634 * CHUNK * abs(at - e) > 150
            assert at == want or faded                                  # all there is, or all that is not 0
