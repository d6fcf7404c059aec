"""Rotary calls on the host (CPU only): the plan's values and every refusal ahead of a launch."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rope as orope

A, B = 256, 1 << 40  # aligned addresses, of inputs and outputs, that no refused call reads


@pytest.fixture(scope="module")
def vcs():
    from paper_2607_11185_gb300 import vcs as v
    return v


@pytest.mark.parametrize("d,sections,theta", [(128, (16, 24, 24), 1e6), (64, (8, 12, 12), 1e4), (64, None, 10000.0),
                                              (16, (8,), 2.5), (256, (32, 32, 32, 32), 1e7)])
def test_plan(vcs, d, sections, theta):
    rope = vcs.rope_plan(d, sections, theta)
    inv, axis = orope.frequencies(d, sections or (d // 2,), theta)
    assert (rope.rot_dim, rope.num_axes, rope.interleaved) == (d, len(sections or (0,)), 0)
    assert np.allclose(rope.inv_freq[:d // 2], inv, rtol=1e-15) and rope.pair_axis[:d // 2] == axis.tolist()


def test_plan_refusals(vcs):
    for kw in (dict(d=64, sections=(8, 12, 13)), dict(d=64, sections=(40, -8)), dict(d=24), dict(d=512), dict(d=0),
               dict(d=64, theta=0.0), dict(d=64, theta=float("nan")), dict(d=64, theta=float("inf")),
               dict(d=64, sections=(8, 8, 8, 4, 4)), dict(d=64, sections=())):
        with pytest.raises(vcs.VcsError):
            vcs.rope_plan(**kw)
    assert vcs.vcs_rope_init(None, 64, 1, (32,), 1e4, 0) == 1


def test_plan_refuses_numbers_past_32_bits(vcs):
    wide = 1 << 32
    for kw in (dict(d=64, rot_dim=wide + 64, sections=(32,)), dict(d=64, sections=(wide + 32,)),
               dict(d=64, sections=(wide + 8, 12, 12)), dict(d=64, sections=(8 - wide, 12, 12)), dict(d=wide + 64)):
        with pytest.raises(vcs.VcsError):
            vcs.rope_plan(**kw)


def test_positions_refusals(vcs):
    def f(cu=A, ns=1, nt=10, src=A, img=A, txt=A, grid=A, steps=4, pos=A):
        return vcs.vcs_stream_positions(cu, ns, nt, src, img, txt, grid, steps, pos, None, 0)
    for kw in (dict(cu=None), dict(ns=-1), dict(nt=-1), dict(src=None), dict(img=None), dict(txt=None),
               dict(grid=None), dict(steps=-1), dict(steps=0), dict(pos=None), dict(ns=0)):
        assert f(**kw) == 1, kw
    assert f(nt=1 << 31) == 4 and f(steps=1 << 31) == 4


def test_rope_refusals(vcs):
    good = vcs.rope_plan(64, (8, 12, 12))

    def bad(**kw):
        r = vcs.VcsRope()
        ctypes.memmove(ctypes.addressof(r), ctypes.addressof(good), ctypes.sizeof(r))
        for k, v in kw.items():
            if isinstance(v, tuple):
                getattr(r, k)[v[0]] = v[1]
            else:
                setattr(r, k, v)
        return r

    def fwd(q=A, k=A, v=A, tt=10, gat=A, pos=A, nt=12, hq=2, hkv=1, d=64, rope=good, oq=B, ok=2 * B, ov=3 * B):
        return vcs.vcs_gather_rope(q, k, v, tt, gat, pos, nt, hq, hkv, d, rope, oq, ok, ov, None, 0)

    def bwd(q=A, k=A, v=A, nt=12, pos=A, off=A, tok=A, tt=10, hq=2, hkv=1, d=64, rope=good, oq=B, ok=2 * B, ov=3 * B):
        return vcs.vcs_gather_rope_bwd(q, k, v, nt, pos, off, tok, tt, hq, hkv, d, rope, oq, ok, ov, None, 0)

    ropes = [bad(rot_dim=24), bad(rot_dim=0), bad(rot_dim=512), bad(num_axes=0), bad(num_axes=5),
             bad(pair_axis=(5, 3)), bad(pair_axis=(31, -1)), bad(inv_freq=(2, float("nan"))),
             bad(inv_freq=(0, float("inf")))]
    for f in (fwd, bwd):
        for kw in [dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(oq=None), dict(ok=None),
                   dict(ov=None), dict(nt=-1), dict(tt=-1), dict(hq=0), dict(hkv=0), dict(d=0), dict(rope=None),
                   dict(q=A + 8), dict(ov=B + 2), *(dict(rope=r) for r in ropes)]:
            assert f(**kw) == 1, kw
        for kw in (dict(d=60), dict(d=48), dict(d=264), dict(hq=65536), dict(hkv=65536)):
            assert f(**kw) == 2, kw
        assert f(nt=1 << 31) == 4 and f(tt=1 << 31) == 4
    for f, rows, out in ((fwd, 10, 12), (bwd, 12, 10)):     # outputs that reach into an input, by a row or whole
        for kw in (dict(oq=A), dict(ok=A), dict(ov=A), dict(q=B - 256, oq=B), dict(v=B + (out - 1) * 256, oq=B),
                   dict(q=2 * B - rows * 256 + 128), dict(k=3 * B + out * 128 - 16)):
            assert f(**kw) == 1, kw
    assert fwd(gat=None) == 1                       # no map: as many rows as tokens
    assert bwd(off=None) == 1 and bwd(tok=None) == 1 and bwd(off=None, tok=None) == 1


def test_inverse_refusals(vcs):
    nb = vcs.vcs_gather_inverse_workspace_size(10)

    def f(gat=A, nt=10, tt=5, off=A, tok=A, ws=A, n=nb):
        return vcs.vcs_gather_inverse(gat, nt, tt, off, tok, None, ws, n, 0)
    for kw in (dict(gat=None), dict(nt=-1), dict(tt=-1), dict(off=None), dict(tok=None)):
        assert f(**kw) == 1, kw
    assert f(tt=(1 << 31) - 1) == 4 and f(nt=1 << 31) == 4 and f(nt=(1 << 31) - 4096) == 4
    assert f(ws=None) == 8 and f(n=nb - 1) == 8 and f(ws=A + 16) == 8
    assert vcs.vcs_gather_inverse_workspace_size(-1) == vcs.vcs_gather_inverse_workspace_size(0)


def test_wrappers_refuse_what_the_kernels_would_misread(vcs):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    rope = vcs.rope_plan(64)
    for call in (lambda: vcs.stream_positions(i, i, i, i, torch.zeros(4, 3, dtype=torch.int32)),
                 lambda: vcs.gather_rope(x, x, x, i, i[None], rope), lambda: vcs.gather_inverse(i, 4),
                 lambda: vcs.gather_rope_bwd(x, x, x, i[None], None, None, rope)):
        with pytest.raises(ValueError, match="not a CUDA device"):
            call()
