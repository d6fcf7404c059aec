"""Windowed attention on the host (CPU only): refusals, workspaces, and the split of the sinks' key tiles."""
import os
import re

import numpy as np
import pytest
import torch

from tests.test_kernel_waits import CSRC, read

A = 256


@pytest.fixture(scope="module")
def vcs():
    from paper_2607_11185_gb300 import vcs as v
    return v


def test_refusals(vcs):
    big = 1 << 40

    def fwd(q=A, k=A, v=A, cu=A, ns=1, nt=10, mx=10, hq=2, hkv=1, d=64, w=4, s=0, o=A, lse=A, ws=A, n=big):
        return vcs.vcs_attn_fwd_window(q, k, v, cu, ns, nt, mx, hq, hkv, d, 0.0, w, s, o, lse, ws, n, 0)

    def bwd(q=A, k=A, v=A, cu=A, ns=1, nt=10, mx=10, hq=2, hkv=1, d=64, w=4, s=0, o=A, lse=A, ws=A, n=big, do=A, dq=A,
            dk=A, dv=A):
        return vcs.vcs_attn_bwd_window(q, k, v, o, lse, do, cu, ns, nt, mx, hq, hkv, d, 0.0, w, s, dq, dk, dv, ws, n, 0)

    for f in (fwd, bwd):
        for kw in (dict(w=0), dict(w=-3), dict(s=-1), dict(q=None), dict(k=None), dict(v=None), dict(cu=None),
                   dict(ns=-1), dict(nt=-1), dict(mx=-1), dict(hq=0), dict(hkv=0), dict(o=None), dict(lse=None),
                   dict(q=A + 8), dict(o=A + 8), dict(lse=A + 4)):
            assert f(**kw) == 1, kw
        for kw in (dict(d=96), dict(d=256), dict(hq=3, hkv=2), dict(hq=65536), dict(hq=1, hkv=2)):
            assert f(**kw) == 2, kw
        assert f(nt=1 << 31) == 4
        for kw in (dict(ws=None), dict(ws=A + 16), dict(n=255)):
            assert f(**kw) == 8, kw
    for kw in (dict(do=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dv=A + 8)):
        assert bwd(**kw) == 1, kw
    need = vcs.vcs_attn_bwd_window_workspace_size(1, 50_000, 50_000, 2, 1, 64, 128, 4)
    assert bwd(nt=50_000, mx=50_000, w=128, s=4, n=need - 1) == 8


def chunk_of(G, mx, w, s):
    """The documented rule: row tiles of a part, None where sink tiles are not split."""
    w, s, rows = min(w, mx), min(s, mx), -(-mx // 128)
    chunk = max((w + 126) // 128 + 1, 2 * -(-s // 128), -(-28 // G))
    return chunk if 0 < s <= 8 * 128 and 2 * chunk - chunk // 3 <= rows else None


def test_backward_workspace(vcs):
    up = lambda x: -(-x // 256) * 256  # noqa: E731
    for ns, nt, mx, hq, hkv, d, w, s in ((1, 50_000, 50_000, 2, 1, 64, 128, 4), (3, 9000, 4000, 8, 2, 128, 256, 300),
                                         (7, 246_616, 46_176, 40, 8, 128, 1024, 4), (1, 70_000, 70_000, 4, 4, 64, 64, 0),
                                         (2, 100, 64, 4, 1, 64, 1, 1), (1, 50_000, 50_000, 2, 1, 64, 128, 2000)):
        chunk = chunk_of(hq // hkv, mx, w, s)
        more = up(hkv * -(-min(s, mx) // 128) * 2 * (nt // (chunk * 128) + 1) * 2 * 128 * d * 4) if chunk else 0
        assert vcs.vcs_attn_bwd_window_workspace_size(ns, nt, mx, hq, hkv, d, w, s) == \
            vcs.vcs_attn_bwd_workspace_size(ns, nt, mx, hq, hkv, d) + more


def test_workspaces_follow_the_tokens_where_the_bound_is_loose(vcs):
    # max_seqlen is a bound; no segment is longer than all tokens
    for nt in (0, 1, 300, 9000, 50_000):
        for mx in (nt + 1, 10 * nt + 129, 2 ** 31 - 128, 2 ** 31 - 1):
            for w, s in ((64, 4), (1024, 300), (2 ** 31 - 1, 5), (1, 2 ** 31 - 1)):
                assert vcs.vcs_attn_bwd_window_workspace_size(1, nt, mx, 4, 1, 64, w, s) == \
                    vcs.vcs_attn_bwd_window_workspace_size(1, nt, nt, 4, 1, 64, w, s), (nt, mx, w, s)
            assert vcs.vcs_attn_bwd_workspace_size(1, nt, mx, 4, 1, 64) == vcs.vcs_attn_bwd_workspace_size(1, nt, nt, 4, 1, 64)
            assert vcs.vcs_attn_fwd_workspace_size(1, nt, mx, 4, 1, 64) == vcs.vcs_attn_fwd_workspace_size(1, nt, nt, 4, 1, 64)


def test_slots_of_split_tiles_are_distinct():
    # the kernel's rule: part p of a segment of more than `chunk` row tiles takes slot
    # 2 ((start + 128 chunk p) / (128 chunk)) + (p == 0), below 2 (tokens / (128 chunk) + 1)
    rng = np.random.default_rng(0)
    for _ in range(300):
        chunk = int(rng.integers(1, 5))
        lens = rng.choice([0, 1, 100, 128 * chunk, 128 * chunk + 1, 128 * chunk + 130, 1000, 3000], size=20)
        ends, seen = np.cumsum(lens), set()
        for start, n in zip(ends - lens, lens):
            rows = -(-int(n) // 128)
            if rows <= chunk:
                continue
            for p in range(-(-rows // chunk)):
                slot = 2 * ((int(start) + p * chunk * 128) // (chunk * 128)) + (p == 0)
                assert slot not in seen and slot < 2 * (int(ends[-1]) // (chunk * 128) + 1)
                seen.add(slot)


def test_parts_of_sink_tiles_cover_every_row_tile_once():
    # the kernel's rules: which key tile and part a CTA takes, and which row tiles a part has
    rng = np.random.default_rng(1)
    for _ in range(400):
        longest, G = int(rng.integers(1, 40_000)), int(rng.choice([1, 2, 5, 7, 8, 40]))
        window, sinks = int(rng.choice([1, 64, 128, 200, 1024, 5000])), int(rng.integers(1, 1100))
        chunk, tiles, rows = chunk_of(G, longest, window, sinks), -(-min(sinks, longest) // 128), -(-longest // 128)
        if chunk is None:
            continue
        parts = (rows + chunk // 3) // chunk
        assert parts >= 2
        seen = set()
        for x in range(rows + tiles * (parts - 1)):
            p, r = divmod(x, tiles + chunk)
            p += 1
            seen.add((x - (parts - 1) * tiles, 0) if p >= parts else (r, p) if r < tiles else
                     ((p - 1) * chunk + r - tiles, 0))
        assert seen == {(n, 0) for n in range(rows)} | {(n, p) for n in range(tiles) for p in range(1, parts)}
        start, slots, nt = 0, set(), longest + 3 * 777
        for length in (longest, 777, 777, 777):  # and shorter segments, of fewer parts or one
            for n in range(min(tiles, -(-length // 128))):
                mine = -(-(length - n * 128) // 128)
                count = max(1, (mine + chunk // 3) // chunk)
                assert count <= parts
                rows_of = []
                for p in range(count):
                    first = mine - (count - p) * chunk if p > 0 else 0
                    rows_of += range(first, mine - (count - 1 - p) * chunk)
                    if count > 1:
                        slot = (n, 2 * ((start + p * chunk * 128) // (chunk * 128)) + (p == 0))
                        assert slot not in slots and slot[1] < 2 * (nt // (chunk * 128) + 1)
                        slots.add(slot)
                assert rows_of == list(range(mine))
            start += length


def test_sizes_for_any_arguments(vcs):
    for hq, hkv in ((0, 1), (1, 0), (-4, 2), (4, -2), (1, 8), (0, 0)):
        vcs.vcs_attn_bwd_window_workspace_size(1, 9000, 9000, hq, hkv, 64, 128, 4)  # returns


def test_no_lane_decides_alone():
    with open(os.path.join(CSRC, "attn_window.cu")) as f:
        src = f.read()
    src = src[src.index("__launch_bounds__(kThreads, 1)"):]
    lone, branches = read(src[src.index("{"):src.index("\n}\n") + 2])
    assert lone == [] and branches == []


def units(G, L, window, sinks):
    """Units of one kv head as the kernel lists them, and the key tiles each of its tiles takes."""
    tiles = -(-L // 128)
    out = []
    for i in range((tiles >> 1) * G + (tiles & 1) * ((G + 1) >> 1)):
        p, r = divmod(i, G)
        half = 2 * p + 1 >= tiles
        pair = r if half else r >> 1
        two = pair < G >> 1
        m0 = 2 * p + (r & 1 if two and not half else 0)
        m1 = m0 if two else m0 + 1
        has1 = two or m1 * 128 < L
        last = m1 if has1 else m0
        lo = max(0, m0 * 128 - window + 1) >> 7
        ns = min((sinks >> 7) + (sinks & 127 != 0), lo)
        nkv = ns + last - lo + 1
        skip = ns if not two and has1 and max(0, m1 * 128 - window + 1) >> 7 > lo and lo * 128 >= sinks else -1
        kt = [j if j < ns else j - ns + lo for j in range(nkv)]
        out.append((2 * pair, m0, kt[:nkv - (last - m0)]))
        if has1:
            out.append((2 * pair + (1 if two else 0), m1, [t for j, t in enumerate(kt) if j != skip]))
    return out


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8])
def test_units_cover_every_row_tile_and_visible_key_once(G):
    for L in (1, 127, 128, 129, 256, 257, 640, 1000):
        for window in (1, 2, 127, 128, 129, 130, 256, 400, 2000):
            for sinks in (0, 1, 127, 128, 129, 300, 5000):
                got = units(G, L, window, sinks)
                tiles = -(-L // 128)
                assert sorted((h, m) for h, m, _ in got) == [(h, m) for h in range(G) for m in range(tiles)]
                for _, m, kt in got:
                    assert len(set(kt)) == len(kt) and kt[-1] == m
                    for t in range(m + 1):  # a tile with a key that a row of the tile sees is among them
                        lo_row = m * 128
                        if t * 128 < sinks or (t + 1) * 128 - 1 > lo_row - window:
                            assert t in kt, (L, window, sinks, m, t)


def test_wrappers_refuse_what_the_kernels_would_misread(vcs):
    x, cu = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="not a CUDA device"):
        vcs.attn_fwd_window(x, x, x, cu, 4, 2)
    with pytest.raises(ValueError, match="not a CUDA device"):
        vcs.attn_bwd_window(x, x, x, x, x, x, cu, 4, 2)


def test_every_declared_call_is_bound(vcs):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "vcs.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(vcs_[a-z0-9_]+)\s*\(", text)) == set(vcs.EXPORTED)
