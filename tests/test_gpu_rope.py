"""GPU parity of the rotary calls: positions and inverse exactly, rotated rows and gradients against fp64.

Tolerances: a result is rounded once to bf16 (half a step, 2^-8 of it).  Before that a rotated pair
(a, b) is off by at most 1e-6 (|a| + |b|): sincospi within 2 ulp of a value below 1 (2.4e-7), its
argument's rounding to 24 bits and to 2^-32 of a turn (1e-7 radians), two roundings of fp32 (1.2e-7).  The
frequency in turns is rounded to 2^-52 of itself, 2^-51 radians a position with the oracle's own angle.
A sum of m copies adds at most m 2^-24 of the terms' sizes.
"""
import numpy as np
import pytest
import torch

from oracle import rope as orope
from oracle import segments as oseg
from paper_2607_11185_gb300 import workloads
from tests.gpu_cases import random_steps

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def _vcs():
    from paper_2607_11185_gb300 import vcs
    return vcs


def dev(*xs):
    return [torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda() for x in xs]


def grids(img, rng, frames=2):
    """A T x H x W for every screenshot size."""
    out = np.zeros((len(img), 3), np.int32)
    for i, n in enumerate(img):
        if n == 0:
            continue
        t = int(rng.choice([x for x in range(1, frames + 1) if n % x == 0]))
        h = int(rng.choice([x for x in range(1, n // t + 1) if (n // t) % x == 0]))
        out[i] = t, h, n // t // h
    return out


# ------------------------------------------------------------------ positions
def check_positions(lay, img, txt, grid):
    vcs = _vcs()
    pos = vcs.stream_positions(*dev(lay["cu_seqlens"], lay["tok_src_step"], img, txt, grid))
    want = orope.positions(lay["cu_seqlens"], lay["tok_src_step"], img, txt, grid)
    assert pos.shape == (3, len(lay["tok_src_step"])) and np.array_equal(pos.cpu().numpy(), want)


@pytest.mark.parametrize("seed", range(12))
def test_positions_random(seed):
    cu, img, txt = random_steps(seed, max_traj=6, max_T=30)
    lay = oseg.build(cu, img, txt, seed % 4 + 1, seed % 3)
    check_positions(lay, img, txt, grids(img, np.random.default_rng(seed)))


@pytest.mark.parametrize("name,window,keep", [("tiny", 2, 0), ("traj8_w3", 3, 0), ("traj8_w3", 1, 1)])
def test_positions_workloads(name, window, keep):
    cu, img, txt = workloads.draw_steps(workloads.WORKLOADS[name])
    check_positions(oseg.build(cu, img, txt, window, keep), img, txt, grids(img, np.random.default_rng(3)))


def test_positions_many_steps_and_chunks():
    # one segment of 700 steps (three tiles of steps) and 30,000 tokens (four chunks), one of 5 tokens
    rng = np.random.default_rng(5)
    img = rng.integers(0, 60, size=705).astype(np.int32)
    txt = rng.integers(0, 30, size=705).astype(np.int32)
    cu = np.array([0, 700, 705], np.int32)
    check_positions(oseg.build(cu, img, txt, 1000, 0), img, txt, grids(img, rng))


def test_positions_of_a_segment_of_thousands_of_steps():
    # 20,000 short steps in one segment (79 tiles of steps, 37 chunks of tokens), one of a single step behind it
    rng = np.random.default_rng(6)
    img, txt = (rng.integers(0, most, size=20_001).astype(np.int32) for most in (21, 11))
    img[-1], txt[-1] = 12, 3
    check_positions(oseg.build(np.array([0, 20_000, 20_001], np.int32), img, txt, 30_000, 0), img, txt, grids(img, rng))


def test_positions_device_checks():
    vcs = _vcs()
    img, txt, grid = [6, 4], [2, 1], [[1, 2, 3], [1, 1, 4]]
    cu, src = [0, 13], [0] * 8 + [1] * 5
    vcs.stream_positions(*dev(cu, src, img, txt, grid))
    for bad in (dict(grid=[[1, 2, 4], [1, 1, 4]]), dict(grid=[[-1, -2, 3], [1, 1, 4]]),
                dict(grid=[[1, 65536, 65536], [1, 1, 4]]), dict(src=[0] * 7 + [1] * 6), dict(src=[2] * 13),
                dict(src=[-1] * 13), dict(src=[1] * 5 + [0] * 8), dict(src=[0, 1, 0, 1, 0, 1, 0, 1, 0, 1, 0, 1, 1]),
                dict(cu=[0, 12]), dict(cu=[1, 13]), dict(cu=[0, 14])):
        x = dict(cu=cu, src=src, img=img, txt=txt, grid=grid) | bad
        with pytest.raises(vcs.VcsError) as e:
            vcs.stream_positions(*dev(x["cu"], x["src"], x["img"], x["txt"], x["grid"]))
        assert e.value.status == 6, bad


@pytest.mark.parametrize("src", [
    [5] * 4 + [3] * 8 + [5] * 20, [5] + [0] * 11 + [5] * 20, [9] + [2] * 299 + [9] * 300, [9] * 100 + [3] * 60 + [9] * 300,
    [9] * 40 + [0] * 260 + [9] * 20, [7] * 2 + [6] * 998 + [7] * 700, [8] * 10 + [2] * 9000 + [8] * 20_000])
def test_positions_that_start_out_of_order(src):
    # the tokens that stand in for a run of the first step are its whole number, but it begins behind them
    vcs = _vcs()
    steps = np.arange(10)
    img = np.where(steps == 5, 12, 280).astype(np.int32)
    txt = np.where(steps == 5, 8, 20).astype(np.int32)
    txt[7], txt[8], txt[0] = 420, 20_000, 4
    grid = np.stack([np.ones(10, int), np.where(steps == 5, 3, 14), np.where(steps == 5, 4, 20)], 1)
    for head in (0, 4):  # alone, and behind a segment that is in order
        cu = [0, head, head + len(src)] if head else [0, len(src)]
        with pytest.raises(vcs.VcsError) as e:
            vcs.stream_positions(*dev(cu, [0] * head + src, img, txt, grid))
        assert e.value.status == 6


def test_positions_empty():
    vcs = _vcs()
    i = torch.zeros(0, dtype=torch.int32, device="cuda")
    pos = vcs.stream_positions(torch.zeros(1, dtype=torch.int32, device="cuda"), i, i, i, i.view(0, 3))
    assert pos.shape == (3, 0)


# ------------------------------------------------------------------ inverse map
@pytest.mark.parametrize("n,t", [(0, 0), (0, 7), (1, 1), (1, 5000), (31, 3), (4096, 1), (4097, 255), (9000, 256),
                                 (50_000, 70_000), (300_000, 65_535), (20_000, 17_000_000)])
def test_inverse(n, t):
    vcs = _vcs()
    rng = np.random.default_rng(n + t)
    gat = rng.integers(0, max(t, 1), size=n)
    off, tok = vcs.gather_inverse(*dev(gat), t)
    order = np.argsort(gat, kind="stable")
    assert np.array_equal(tok.cpu().numpy(), order)
    assert np.array_equal(off.cpu().numpy(), np.searchsorted(gat[order], np.arange(t + 1)))


@pytest.mark.parametrize("kind", ["stretches", "one token", "descending", "bad", "pairs"])
@pytest.mark.parametrize("n,t", [(4097, 9000), (100_003, 8191), (100_003, 1_900_000), (100_003, 3_000_001), (5_000_011, 1_200_000),
                                 (5_000_011, 40)])
def test_inverse_of_runs(n, t, kind):
    """Stretches of consecutive tokens (a layout's map), and maps whose runs are longest, shortest, or out of range."""
    vcs = _vcs()
    rng = np.random.default_rng(n + t)
    i = np.arange(n)
    if kind == "stretches":
        cuts = np.unique(rng.integers(0, n, n // 300))
        start = rng.integers(0, t, len(cuts) + 1)
        part = np.searchsorted(cuts, i, side="right")
        gat = (start[part] + i - np.concatenate([[0], cuts])[part]) % t
    elif kind == "one token":
        gat = np.full(n, t - 1)
    elif kind == "descending":
        gat = (n - 1 - i) % t
    elif kind == "bad":
        gat = np.where(i % 1000 < 300, i % t, np.where(i % 2 == 0, -1 - i, t + i))
    else:
        gat = i // 2 % t
    off, tok = vcs.gather_inverse(*dev(gat), t, check=False)
    key = np.where((gat < 0) | (gat >= t), t, gat)
    order = np.argsort(key, kind="stable")
    assert np.array_equal(tok.cpu().numpy(), order)
    assert np.array_equal(off.cpu().numpy(), np.searchsorted(key[order], np.arange(t + 1)))


def test_inverse_of_a_part_of_a_map():
    vcs = _vcs()
    gat = np.arange(20_001) * 2 // 3
    for cut in (1, 2, 3):
        part = dev(gat)[0][cut:]  # at an address that 16 bytes do not divide
        off, tok = vcs.gather_inverse(part, int(gat[-1]) + 1)
        assert np.array_equal(tok.cpu().numpy(), np.arange(len(gat) - cut))
        assert np.array_equal(off.cpu().numpy(), np.searchsorted(gat[cut:], np.arange(gat[-1] + 2)))


def test_inverse_captured_replayed_and_beside_another():
    vcs = _vcs()
    t = 20_000
    maps = [dev((np.arange(60_000) * 7 // 8 + c) % t)[0] for c in (0, 5)] + dev(np.full(60_000, 3))
    want = []
    for m in maps:
        key = m.cpu().numpy()
        order = np.argsort(key, kind="stable")
        want.append((np.searchsorted(key[order], np.arange(t + 1)), order))

    def check(got, i):
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want[i])), i
    gat = maps[0].clone()
    vcs.gather_inverse(gat, t)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = vcs.gather_inverse(gat, t, check=False)
    for i in (2, 0, 1, 2):  # one token's 60,000 copies before and behind others: nothing is left of a replay
        gat.copy_(maps[i])
        g.replay()
        check(got, i)
    sides = [torch.cuda.Stream() for _ in maps]
    torch.cuda.synchronize()
    outs = [vcs.gather_inverse(m, t, stream=x, check=False) for x, m in list(zip(sides, maps)) * 3]
    torch.cuda.synchronize()
    for k, o in enumerate(outs):
        check(o, k % 3)


@pytest.mark.parametrize("n", [5, 5000])
def test_inverse_of_no_tokens(n):
    vcs = _vcs()
    off, tok = vcs.gather_inverse(torch.zeros(n, dtype=torch.int32, device="cuda"), 0, check=False)
    assert off.tolist() == [0] and tok.tolist() == list(range(n))


def test_inverse_of_a_layout_and_bad_entries():
    vcs = _vcs()
    cu, img, txt = random_steps(3)
    lay = oseg.build(cu, img, txt, 2, 1)
    t = int(img.sum() + txt.sum())
    off, tok = vcs.gather_inverse(*dev(lay["tok_gather"]), t)
    want = orope.inverse(lay["tok_gather"], t)
    assert np.array_equal(off.cpu().numpy(), want[0]) and np.array_equal(tok.cpu().numpy(), want[1])
    bad = np.array([2, -1, 0, 7, 2, 5, -2 ** 31])
    with pytest.raises(vcs.VcsError) as e:
        vcs.gather_inverse(*dev(bad), 5)
    assert e.value.status == 6
    off, tok = vcs.gather_inverse(*dev(bad), 5, check=False)
    assert off.tolist() == [0, 1, 1, 3, 3, 3] and tok.tolist() == [2, 0, 4, 1, 3, 5, 6]


# ------------------------------------------------------------------ rotation
def bound(ref, size, pos, copies=1):
    far = np.abs(np.asarray(pos, np.float64)).max() if np.size(pos) else 0.0
    slip = (1e-6 + far * 2.0 ** -51 + copies * 2.0 ** -24) * size
    return HALF * (np.abs(ref) + slip) + slip


def pair_size(x, rot, interleaved):
    """|a| + |b| of the pair each dim is in, and the dim's own size where it is not turned."""
    y = np.abs(x).copy()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = y[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y


def rows(seed, n, h, d):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((n, h, d), generator=g, device="cuda").bfloat16()


CASES = [  # hq, hkv, d, rot, sections, interleaved
    (2, 1, 64, 64, (8, 12, 12), False), (2, 1, 64, 64, (8, 12, 12), True), (28, 4, 128, 128, (16, 24, 24), False),
    (5, 5, 128, 96, (16, 16, 16), False), (3, 3, 128, 48, (24,), True), (1, 1, 16, 16, (4, 4), False),
    (1, 1, 24, 16, (8,), True), (7, 1, 256, 256, (32, 32, 32, 32), False), (2, 2, 256, 240, (60, 60), True),
    (3, 1, 72, 64, (0, 32), False)]


@pytest.mark.parametrize("hq,hkv,d,rot,sections,inter", CASES)
@pytest.mark.parametrize("n,t", [(1, 1), (37, 20), (700, 90)])
def test_gather_rope_and_backward(hq, hkv, d, rot, sections, inter, n, t):
    vcs = _vcs()
    rng = np.random.default_rng(n + d)
    gat = rng.integers(0, t, size=n)
    pos = rng.integers(0, 70_000, size=(len(sections), n))
    rope = vcs.rope_plan(d, sections, 1e6, rot_dim=rot, interleaved=inter)
    inv, axis = orope.frequencies(rot, sections, 1e6)
    q, k, v = rows(1, t, hq, d), rows(2, t, hkv, d), rows(3, t, hkv, d)
    got = vcs.gather_rope(q, k, v, *dev(gat, pos), rope)
    assert torch.equal(got[2], v[torch.from_numpy(gat).cuda()])
    for x, y in ((q, got[0]), (k, got[1])):
        src = x.double().cpu().numpy()[gat]
        ref = orope.rotate(src, pos, inv, axis, inter)
        assert (np.abs(y.double().cpu().numpy() - ref) <= bound(ref, pair_size(src, rot, inter), pos)).all()
    dq, dk, dv = rows(4, n, hq, d), rows(5, n, hkv, d), rows(6, n, hkv, d)
    off, tok = vcs.gather_inverse(*dev(gat), t)
    back = vcs.gather_rope_bwd(dq, dk, dv, *dev(pos), off, tok, rope)
    copies = int(np.bincount(gat).max())
    for x, y, turn in ((dq, back[0], True), (dk, back[1], True), (dv, back[2], False)):
        src = x.double().cpu().numpy()
        ref = orope.rotate(src, pos, inv, axis, inter, back=True) if turn else src
        size = pair_size(src, rot, inter) if turn else np.abs(src)
        ref, size = orope.scatter(ref, gat, t), orope.scatter(size, gat, t)
        assert (np.abs(y.double().cpu().numpy() - ref) <= bound(ref, size, pos, copies)).all()
    again = vcs.gather_rope_bwd(dq, dk, dv, *dev(pos), off, tok, rope)
    assert all(torch.equal(a, b) for a, b in zip(back, again))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(160, 144), (160, 160), (176, 176), (192, 176), (192, 192), (256, 144), (256, 160),
                                   (256, 192), (256, 208)])
@pytest.mark.parametrize("hq,hkv,n,t", [(1, 1, 1, 1), (3, 1, 700, 90), (1, 1, 40_000, 39_000), (28, 4, 300, 90)])
def test_heads_of_128_to_256_rotated_dims(hq, hkv, n, t, d, rot, inter):
    # 65 to 104 pairs, with a row and (40,000 short rows) several a warp
    a = rot // 8
    test_gather_rope_and_backward(hq, hkv, d, rot, (a, 2 * a - 8, rot // 2 - 3 * a + 8), inter, n, t)


@pytest.mark.parametrize("inter", [False, True])
def test_identity_map_any_position(inter):
    # no map: row n is token n; positions of any int32, exact angles far out and negative ones
    vcs = _vcs()
    pos = np.array([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123_456_789, 1000, -77, 5, 6, 7]])
    n = pos.shape[1]
    rope = vcs.rope_plan(64, (32,), 1e4, interleaved=inter)
    inv, axis = orope.frequencies(64, (32,), 1e4)
    q, k, v = rows(1, n, 4, 64), rows(2, n, 2, 64), rows(3, n, 2, 64)
    got = vcs.gather_rope(q, k, v, None, *dev(pos), rope)
    back = vcs.gather_rope_bwd(q, k, v, *dev(pos), None, None, rope)
    assert torch.equal(got[2], v) and torch.equal(back[2], v) and torch.equal(got[0][0], q[0])
    for x, y, z in ((q, got[0], back[0]), (k, got[1], back[1])):
        src = x.double().cpu().numpy()
        for res, b in ((y, False), (z, True)):
            ref = orope.rotate(src, pos, inv, axis, inter, back=b)
            assert (np.abs(res.double().cpu().numpy() - ref) <= bound(ref, pair_size(src, 64, inter), pos)).all()


def test_changed_frequencies_and_axes():
    # axes by turns, a frequency of 0, a negative one and one of many turns a position
    vcs = _vcs()
    rng = np.random.default_rng(8)
    rope = vcs.rope_plan(32, (6, 5, 5), 100.0)
    inv, axis = orope.frequencies(32, (6, 5, 5), 100.0)
    axis = np.arange(16) % 3
    inv[3], inv[5], inv[7], inv[9] = 0.0, -0.25, 40.0, -1e-300
    for i in range(16):
        rope.inv_freq[i], rope.pair_axis[i] = inv[i], int(axis[i])
    pos = rng.integers(0, 430, size=(3, 50))
    x = rows(1, 50, 2, 32)
    got = vcs.gather_rope(x, x, x, None, *dev(pos), rope)
    src = x.double().cpu().numpy()
    ref = orope.rotate(src, pos, inv, axis)
    assert (np.abs(got[0].double().cpu().numpy() - ref) <= bound(ref, pair_size(src, 32, False), 40 * pos)).all()


@pytest.mark.parametrize("inter", [False, True])
def test_negative_frequencies_turn_the_other_way(inter):
    # -f at n is f at -n, bit for bit, however far n is and however small f
    vcs = _vcs()
    rng = np.random.default_rng(9)
    n = 4000
    pos = rng.integers(-2 ** 31 + 1, 2 ** 31, size=(1, n))
    one, other = (vcs.rope_plan(128, (64,), 1e9, interleaved=inter) for _ in range(2))
    for i in range(64):
        other.inv_freq[i] = -one.inv_freq[i]
    x = rows(1, n, 8, 128)
    got, want = (vcs.gather_rope(x, x, x, None, *dev(p), r) for p, r in ((pos, other), (-pos, one)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_many_copies_and_none():
    # a token of 1,000 copies, some of 7 to 9 (around a warp's batch of angles), some of none
    vcs = _vcs()
    gat = np.concatenate([np.full(1000, 3), np.repeat([1, 5, 6], [7, 8, 9]), [9]])
    n, t = len(gat), 12
    gat = np.random.default_rng(0).permutation(gat)
    pos = np.random.default_rng(1).integers(0, 5000, size=(3, n))
    rope = vcs.rope_plan(64, (8, 12, 12), 1e6)
    inv, axis = orope.frequencies(64, (8, 12, 12), 1e6)
    dq, dk, dv = rows(4, n, 3, 64), rows(5, n, 1, 64), rows(6, n, 1, 64)
    back = vcs.gather_rope_bwd(dq, dk, dv, *dev(pos), *vcs.gather_inverse(*dev(gat), t), rope)
    for x, y, turn in ((dq, back[0], True), (dk, back[1], True), (dv, back[2], False)):
        src = x.double().cpu().numpy()
        ref = orope.scatter(orope.rotate(src, pos, inv, axis, back=True) if turn else src, gat, t)
        size = orope.scatter(pair_size(src, 64, False), gat, t)
        assert (np.abs(y.double().cpu().numpy() - ref) <= bound(ref, size, pos, 1000)).all()
        assert not y[[0, 2, 4, 7, 8, 10, 11]].any()
    assert torch.equal(back[2][9], dv[int(np.nonzero(gat == 9)[0][0])])


def test_one_copy_keeps_the_bits_of_v():
    vcs = _vcs()
    v = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), 1e-40, -1e-40, 3.0, -5.0] * 2).bfloat16().cuda().view(1, 1, 16)
    pos = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    rope = vcs.rope_plan(16)
    x = torch.ones_like(v)
    for got in (vcs.gather_rope(x, x, v, pos[0], pos, rope)[2],
                vcs.gather_rope_bwd(x, x, v, pos, one, pos[0], rope)[2]):
        assert torch.equal(got.view(torch.int16), v.view(torch.int16))


def test_device_checks_leave_rows_out():
    vcs = _vcs()
    x = rows(1, 6, 2, 64)
    rope = vcs.rope_plan(64)
    gat, pos = dev([0, 6, 2, -1, 5], np.zeros((1, 5)))
    with pytest.raises(vcs.VcsError) as e:
        vcs.gather_rope(x, x, x, gat, pos, rope)
    assert e.value.status == 6
    out = [torch.full((5, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    assert vcs.vcs_gather_rope(x, x, x, 6, gat, pos, 5, 2, 2, 64, rope, *out, None) == 0
    for o in out:
        assert torch.equal(o[[0, 2, 4]], x[[0, 2, 5]]) and (o[[1, 3]] == 7).all()
    y, pos6 = rows(2, 6, 2, 64), torch.zeros((1, 6), dtype=torch.int32, device="cuda")
    for off, tok in (([0, 2, 7, 7], [0, 1, 2, 3, 4, 5]), ([0, 2, 1, 6], [0, 1, 2, 3, 4, 5]), ([-1, 2, 3, 6], [0, 1, 2, 3, 4, 5]),
                     ([0, 2, 3, 6], [0, 6, 2, 3, 4, 5]), ([0, 2, 3, 6], [0, -1, 2, 3, 4, 5])):
        with pytest.raises(vcs.VcsError) as e:
            vcs.gather_rope_bwd(y, y, y, pos6, *dev(off, tok), rope)
        assert e.value.status == 6, (off, tok)
    got = vcs.gather_rope_bwd(y, y, y, pos6, *dev([0, 2, 3, 6], [0, -1, 2, 3, 4, 9]), rope, check=False)
    assert torch.equal(got[2][0], y[0]) and torch.equal(got[2][1], y[2])
    assert torch.equal(got[2][2], (y[3].float() + y[4].float()).bfloat16())


@pytest.mark.parametrize("inter", [False, True])
def test_rows_past_32_bit_offsets(inter):
    # 2.2 billion elements of q, in and out: rows at both ends and around element 2^31 are those of a call on them alone
    vcs = _vcs()
    n = 2 ** 23 + 300_000
    rope = vcs.rope_plan(64, (8, 12, 12), 1e6, interleaved=inter)
    q, k, v = rows(1, n, 4, 64), rows(2, n, 1, 64), rows(3, n, 1, 64)
    g = torch.Generator(device="cuda").manual_seed(4)
    pos = torch.randint(0, 100_000, (3, n), generator=g, device="cuda", dtype=torch.int32)
    back_to_front = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    off, tok = vcs.gather_inverse(back_to_front, n)
    there = vcs.gather_rope(q, k, v, back_to_front, pos, rope)
    back = vcs.gather_rope_bwd(q, k, v, pos, off, tok, rope)
    for a, b in ((0, 1000), (2 ** 23 - 500, 2 ** 23 + 500), (n - 1000, n)):
        at = slice(n - b, n - a)  # the rows' other ends, in reverse
        flip = [x[at].flip(0).contiguous() for x in (q, k, v)]
        want = vcs.gather_rope(*flip, None, pos[:, a:b].contiguous(), rope)
        assert all(torch.equal(x[a:b], y) for x, y in zip(there, want))
        want = vcs.gather_rope_bwd(*flip, pos[:, at].flip(1).contiguous(), None, None, rope)
        assert all(torch.equal(x[a:b], y) for x, y in zip(back, want))


def test_wrappers_refuse_other_layouts():
    vcs = _vcs()
    rope = vcs.rope_plan(64)
    x, pos = rows(1, 6, 2, 64), torch.zeros((1, 6), dtype=torch.int32, device="cuda")
    gat = torch.zeros(6, dtype=torch.int32, device="cuda")
    for bad in ((x.float(), x, x, gat, pos), (x, x[:5], x, gat, pos), (x, x, x[:, :1], gat, pos),
                (x, x, x, gat.long(), pos), (x, x, x, gat, pos[:, :5]), (x, x, x, gat, pos.repeat(3, 1)),
                (rows(1, 12, 2, 64)[::2], x, x, gat, pos), (x, x.cpu(), x, gat, pos), (x, x, x, gat, pos.view(6, 1))):
        with pytest.raises(ValueError):
            vcs.gather_rope(*bad, rope)


def test_on_a_stream_and_in_a_graph():
    vcs = _vcs()
    rng = np.random.default_rng(4)
    n, t = 900, 300
    gat, pos = dev(rng.integers(0, t, size=n), rng.integers(0, 999, size=(3, n)))
    rope = vcs.rope_plan(64, (8, 12, 12))
    q, k, v = rows(1, t, 4, 64), rows(2, t, 2, 64), rows(3, t, 2, 64)
    off, tok = vcs.gather_inverse(gat, t)
    want = vcs.gather_rope(q, k, v, gat, pos, rope)
    wantb = vcs.gather_rope_bwd(*want, pos, off, tok, rope)
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)
    side.wait_stream(torch.cuda.current_stream())
    o2 = vcs.gather_inverse(gat, t, stream=side)
    got = vcs.gather_rope(q, k, v, gat, pos, rope, stream=side)
    gotb = vcs.gather_rope_bwd(*got, pos, *o2, rope, stream=side.cuda_stream)
    assert all(torch.equal(a, b) for a, b in zip((*got, *gotb, *o2), (*want, *wantb, off, tok)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o3 = vcs.gather_inverse(gat, t, check=False)
        got = vcs.gather_rope(q, k, v, gat, pos, rope, check=False)
        gotb = vcs.gather_rope_bwd(*got, pos, *o3, rope, check=False)
    q.copy_(rows(9, t, 4, 64))
    gat.copy_(torch.flip(gat, (0,)))
    g.replay()
    want = vcs.gather_rope(q, k, v, gat, pos, rope)
    wantb = vcs.gather_rope_bwd(*want, pos, *vcs.gather_inverse(gat, t), rope)
    assert all(torch.equal(a, b) for a, b in zip((*got, *gotb), (*want, *wantb)))


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_positions_at_any_alignment(shift):
    # token counts that are and are not multiples of four, buffers off the 16-byte alignment, grids of one row or
    # column and many frames, runs that begin and end inside four tokens
    vcs = _vcs()
    rng = np.random.default_rng(shift)
    grid = np.array([[1, 1, 37], [5, 1, 1], [3, 2, 1], [2, 7, 3], [1, 9, 9], [7, 1, 2], [1, 1, 1]], np.int32)
    grid = grid[rng.integers(0, 7, size=40)]
    img, txt = grid.prod(1).astype(np.int32), rng.integers(0, 7, size=40).astype(np.int32)
    for extra in range(4):
        txt[39] = 5
        lay = oseg.build(np.array([0, 13, 40], np.int32), img, txt, 4, 1)
        txt[39] += (extra - len(lay["tok_src_step"])) % 4
        lay = oseg.build(np.array([0, 13, 40], np.int32), img, txt, 4, 1)
        n = len(lay["tok_src_step"])
        src = torch.zeros(n + 4, dtype=torch.int32, device="cuda")[shift:shift + n]
        src.copy_(torch.from_numpy(lay["tok_src_step"]))
        pos = torch.full((3 * n + 8,), -1, dtype=torch.int32, device="cuda")
        cu, i, t, g = dev(lay["cu_seqlens"], img, txt, grid)
        word = torch.zeros(1, dtype=torch.int32, device="cuda")
        assert vcs.vcs_stream_positions(cu, cu.numel() - 1, n, src, i, t, g, 40, pos[shift:], word) == 0
        want = orope.positions(lay["cu_seqlens"], lay["tok_src_step"], img, txt, grid)
        assert n % 4 == extra and int(word) == 0
        assert np.array_equal(pos[shift:shift + 3 * n].view(3, n).cpu().numpy(), want)
        assert (pos[:shift] == -1).all() and (pos[shift + 3 * n:] == -1).all()
