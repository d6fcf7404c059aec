"""GPU parity of windowed attention against the fp64 oracle.

Elementwise bounds, from the roundings (u = 2^-8, half a step of bf16).  A score is a sum of d products that
are exact in fp32; its error is at most e = 2^-17 scale sum |q||k| (d 2^-24 of the products' sizes), and
exp, the shift by the maximum and the running sum add less than 2^-18 of P.  So P is off by eps =
2 e + 2^-18 of itself, and where it enters a product of the tensor pipe by u more:
  o    (u + eps) sum P|v| + u |o|
  lse  e + 2^-18 (1 + |lse|)
  dv   (u + eps) sum P|do| + u |dv|
  D    from o as stored: sum |do| (error of o);   dP  2^-17 sum |do||v|
  dS   P (error of dP and D) + |dS| (eps + u)
  dq   scale sum (error of dS)|k| + u |dq|, dk likewise over its query rows and heads
with 2^-16 of each sum's terms for its own fp32 additions.  What fp32 cannot hold is flushed: a P, dS or
product below 2^-126 becomes 0, which moves a sum of at most 2^14 terms, each times a factor below 2^8, by
less than 2^-126 2^14 2^8 = 2^-104: TINY.
"""
import numpy as np
import pytest
import torch

from oracle import rope as orope
from oracle import window as owin
from paper_2607_11185_gb300 import workloads
from tests.gpu_cases import cu_from_lengths, steps_to_device

pytestmark = pytest.mark.gpu
U, FP, TINY = 2.0 ** -8, 2.0 ** -16, 2.0 ** -104


def _vcs():
    from paper_2607_11185_gb300 import vcs
    return vcs


def f64(x):
    return x.double().cpu().numpy()


def within(got, want, bound, name):
    over = np.abs(got - want) - bound - TINY
    assert over.size == 0 or over.max() <= 0, (name, int((over > 0).sum()), over.max(), np.unravel_index(over.argmax(), over.shape))


def check(q, k, v, do, lens, window, sinks, scale=0.0, cancels=False):
    vcs = _vcs()
    cu = cu_from_lengths(lens)
    cud, mx = torch.from_numpy(cu).cuda(), int(max(lens, default=0))
    o, lse = vcs.attn_fwd_window(q, k, v, cud, mx, window, sinks, scale)
    got = (o, lse, *vcs.attn_bwd_window(q, k, v, o, lse, do, cud, mx, window, sinks, scale))
    o, lse, dq, dk, dv = (f64(x) for x in got)
    r = owin.attn(q, k, v, cu, window, sinks, do, scale)
    qn, kn, vn, dn = (np.abs(f64(x)) for x in (q, k, v, do))
    sc = scale if scale > 0 else q.shape[2] ** -0.5
    bk, bv = np.zeros_like(kn), np.zeros_like(vn)
    for b, e, h, g, p, ds, dp, dd in r["parts"]:
        err = 2.0 ** -17 * sc * np.where(p > 0, qn[b:e, h] @ kn[b:e, g].T, 0).max(1, keepdims=True)
        eps = 2 * err + 2.0 ** -18
        bo = (U + eps + FP) * (p @ vn[b:e, g]) + U * np.abs(r["o"][b:e, h])
        within(o[b:e, h], r["o"][b:e, h], bo, "o")
        within(lse[h, b:e], r["lse"][h, b:e], err[:, 0] + 2.0 ** -18 * (1 + np.abs(r["lse"][h, b:e])), "lse")
        bd = (dn[b:e, h] * (bo + FP * np.abs(r["o"][b:e, h]))).sum(1, keepdims=True)
        bp = 2.0 ** -17 * (dn[b:e, h] @ vn[b:e, g].T)
        bs = p * (bd + bp) + np.abs(ds) * (eps + U)
        bq = sc * ((bs + FP * np.abs(ds)) @ kn[b:e, g]) + U * np.abs(r["dq"][b:e, h])
        within(dq[b:e, h], r["dq"][b:e, h], bq * (1 + U), "dq")
        bk[b:e, g] += sc * ((bs + FP * np.abs(ds)).T @ qn[b:e, h])
        bv[b:e, g] += ((U + eps + FP) * p).T @ dn[b:e, h]
    within(dk, r["dk"], (bk + U * np.abs(r["dk"])) * (1 + U), "dk")
    within(dv, r["dv"], (bv + U * np.abs(r["dv"])) * (1 + U), "dv")
    for x, name in ((o, "o"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        if name in ("o", "dv") or (window > 1 and max(lens) > 8 and not cancels):
            far, size = np.linalg.norm(x - r[name]), np.linalg.norm(r[name])
            assert far <= 1e-2 * size, (name, far, size)


LENS = [1, 2, 130, 0, 127, 128, 129, 257, 385, 640]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [
    (1, 0), (1, 1), (2, 0), (5, 4), (64, 0), (127, 3), (128, 0), (128, 4), (129, 1), (130, 128), (192, 129), (255, 0),
    (256, 64), (257, 300), (300, 5), (384, 1), (639, 2), (640, 0), (10 ** 9, 0), (3, 10 ** 9), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(d, window, sinks):
    q, k, v, do = workloads.draw_dense(window % 97 + sinks % 89, sum(LENS), 3, 1, d, device="cuda")
    check(q, k, v, do, LENS, window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (2, 2), (4, 2), (5, 1), (7, 1), (8, 4), (16, 2)])
def test_heads(d, hq, hkv):
    lens = [300, 129, 700, 64]
    q, k, v, do = workloads.draw_dense(hq * 10 + hkv, sum(lens), hq, hkv, d, device="cuda")
    check(q, k, v, do, lens, 150, 7)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [1, 2, 127, 128, 129, 255, 256, 257, 383, 384, 385, 513])
def test_lengths(d, length):
    q, k, v, do = workloads.draw_dense(length, length, 2, 1, d, device="cuda")
    check(q, k, v, do, [length], 100, 2)


@pytest.mark.parametrize("d,scale", [(64, 0.5), (128, 0.01), (64, 3.0), (128, 1.0)])
def test_scales_and_large_scores(d, scale):
    lens = [400, 200]
    q, k, v, do = workloads.draw_dense(3, sum(lens), 4, 2, d, device="cuda")
    k[::7] *= 8
    check(q, k, v, do, lens, 140, 4, scale)


def test_rising_and_falling_maxima():
    # Keys whose scores rise along the window (each tile rescales) and sinks far above or below it.  Every key
    # lies along one vector and sum_j dS_ij = 0, so the terms of dq cancel while their roundings, up to u of
    # each, and D's, do not: its error is bound by its terms' sizes, elementwise, and by nothing relative to it.
    lens = [900]
    q, k, v, do = workloads.draw_dense(5, 900, 2, 1, 64, device="cuda")
    q[:] = q.abs() * 0.5
    for sign, sink in ((1.0, 0.0), (-1.0, 12.0), (1.0, -30.0)):
        k = (torch.linspace(-6, 6, 900, device="cuda") * sign)[:, None, None].expand(900, 1, 64).bfloat16().contiguous()
        k[:3] = sink
        check(q, k, v, do, lens, 300, 3, cancels=True)


@pytest.mark.parametrize("hq,hkv,d,lens,window,sinks", [
    (2, 1, 64, [6000], 64, 4),            # three parts of the sinks' tile
    (1, 1, 128, [5000], 200, 130),        # two sink tiles, the second of them partly
    (2, 2, 64, [300, 4100, 20, 2200, 2049, 128], 100, 1),  # split and whole segments side by side
    (3, 1, 128, [2049, 2048, 2177], 130, 128), (1, 1, 64, [4000], 1000, 1024), (1, 1, 64, [4000], 1000, 1025)])
def test_split_sink_tiles(hq, hkv, d, lens, window, sinks):
    q, k, v, do = workloads.draw_dense(len(lens), sum(lens), hq, hkv, d, device="cuda")
    check(q, k, v, do, lens, window, sinks)


@pytest.mark.parametrize("hq,hkv,d,lens,window,sinks", [
    (7, 1, 64, [900, 800, 768, 640, 1200], 100, 4),   # parts of four row tiles and a first of up to six
    (7, 1, 128, [1700, 130], 100, 200),               # two sink tiles, of which the second has a row tile less
    (14, 2, 64, [3000, 900, 1], 200, 300),            # three, in parts of six row tiles
    (28, 1, 64, [1100], 64, 5), (4, 4, 64, [6100], 64, 1)])  # parts of two, and of 28
def test_sink_tiles_in_many_parts(hq, hkv, d, lens, window, sinks):
    q, k, v, do = workloads.draw_dense(len(lens), sum(lens), hq, hkv, d, device="cuda")
    check(q, k, v, do, lens, window, sinks)


@pytest.mark.parametrize("d", [64, 128])
def test_wide_window_equals_causal(d):
    vcs = _vcs()
    lens = [513, 1, 700, 128]
    q, k, v, do = workloads.draw_dense(9, sum(lens), 6, 2, d, device="cuda")
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    o, lse = vcs.attn_fwd(q, k, v, cu, 700)
    for window, sinks in ((700, 0), (1, 700), (350, 400)):
        ow, lw = vcs.attn_fwd_window(q, k, v, cu, 700, window, sinks)
        assert (ow.float() - o.float()).abs().max() <= 2e-2 and (lw - lse).abs().max() <= 1e-4


def test_numbers_past_32_bits():
    # a window, sinks or a bound that an int32 cannot hold is as wide as any that reaches past the longest segment
    vcs = _vcs()
    lens = [300, 40, 700]
    q, k, v, do = workloads.draw_dense(6, sum(lens), 4, 2, 64, device="cuda")
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    wide = [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, 10 ** 30]
    for want_args, calls in (((700, 700, 0), [(700, w, 0) for w in wide]), ((700, 3, 700), [(700, 3, w) for w in wide]),
                             ((700, 90, 4), [(w, 90, 4) for w in wide])):
        o, lse = vcs.attn_fwd_window(q, k, v, cu, *want_args)
        dk, dv = vcs.attn_bwd_window(q, k, v, o, lse, do, cu, *want_args)[1:]
        for args in calls:
            o2, lse2 = vcs.attn_fwd_window(q, k, v, cu, *args)
            dk2, dv2 = vcs.attn_bwd_window(q, k, v, o, lse, do, cu, *args)[1:]
            assert torch.equal(o2, o) and torch.equal(lse2, lse), args
            assert all((a.double() - b.double()).norm() <= 1e-3 * b.double().norm() for a, b in ((dk2, dk), (dv2, dv))), args
    for args in ((700, 5 - 2 ** 32, 0), (700, 5, 5 - 2 ** 32), (700 - 2 ** 32, 5, 0)):
        for f in (lambda: vcs.attn_fwd_window(q, k, v, cu, *args), lambda: vcs.attn_bwd_window(q, k, v, o, lse, do, cu, *args)):
            with pytest.raises(vcs.VcsError) as e:
                f()
            assert e.value.status == 1, args


def test_keys_out_of_sight_do_not_matter():
    # scores that no mask value could stand beside: the largest finite keys, out of the window
    vcs = _vcs()
    q, k, v, do = workloads.draw_dense(4, 1000, 2, 1, 64, device="cuda")
    cu = torch.tensor([0, 1000], dtype=torch.int32, device="cuda")
    o, lse = vcs.attn_fwd_window(q, k, v, cu, 1000, 128, 2)
    k2 = k.clone()
    k2[2:800] = 3e38
    o2, lse2 = vcs.attn_fwd_window(q, k2, v, cu, 1000, 128, 2)
    assert torch.equal(o2[928:], o[928:]) and torch.equal(lse2[:, 928:], lse[:, 928:])
    k2[2:800] = float("nan")
    o2, lse2 = vcs.attn_fwd_window(q, k2, v, cu, 1000, 128, 2)
    assert torch.equal(o2[928:], o[928:]) and torch.equal(lse2[:, 928:], lse[:, 928:])


def test_device_checks():
    vcs = _vcs()
    q, k, v, do = workloads.draw_dense(4, 600, 2, 1, 64, device="cuda")
    lse = torch.zeros((2, 600), device="cuda")
    for cu, mx in (([0, 300, 599], 300), ([1, 300, 600], 300), ([0, 400, 300], 300), ([0, 300, 600], 299),
                   ([0, -5, 600], 600), ([0, 700, 600], 700)):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        for f in (lambda: vcs.attn_fwd_window(q, k, v, c, mx, 64, 2),
                  lambda: vcs.attn_bwd_window(q, k, v, q, lse, do, c, mx, 64, 2)):
            with pytest.raises(vcs.VcsError) as e:
                f()
            assert e.value.status == 6, cu


def test_no_tokens():
    vcs = _vcs()
    q, k = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((0, 1, 64), dtype=torch.bfloat16,
                                                                                    device="cuda")
    for cu in ([0], [0, 0, 0]):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        # an empty tensor has no address: the calls take any other
        buf, ws = torch.zeros(4096, device="cuda"), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        assert vcs.vcs_attn_fwd_window(buf, buf, buf, c, len(cu) - 1, 0, 0, 2, 1, 64, 0.0, 5, 1, buf, buf, ws, 1 << 16) == 0
        assert vcs.vcs_attn_bwd_window(buf, buf, buf, buf, buf, buf, c, len(cu) - 1, 0, 0, 2, 1, 64, 0.0, 5, 1, buf, buf,
                                       buf, ws, 1 << 16) == 0
        torch.cuda.synchronize()
        assert int(ws[0]) == 0
    assert q.numel() == k.numel() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_forward_repeats_bit_for_bit_and_gradients_of_keys(d):
    vcs = _vcs()
    lens = [3000, 500]
    q, k, v, do = workloads.draw_dense(8, sum(lens), 4, 2, d, device="cuda")
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    runs = []
    for _ in range(3):
        o, lse = vcs.attn_fwd_window(q, k, v, cu, 3000, 200, 5)
        runs.append((o, lse, *vcs.attn_bwd_window(q, k, v, o, lse, do, cu, 3000, 200, 5)[1:]))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_long_buffers_past_32_bit_offsets():
    # 2.2 billion elements of q; rows of the last segment and of the first
    vcs = _vcs()
    lens = [200_000, 229_000, 1000]
    n = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (workloads._randn_bf16(g, (n, h, 128), "cuda") for h in (40, 8, 8))
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    o, lse = vcs.attn_fwd_window(q, k, v, cu, max(lens), 200, 3)
    dq, dk, dv = vcs.attn_bwd_window(q, k, v, o, lse, q, cu, max(lens), 200, 3)
    for seg, rows in (((0, 200_000), (0, 250, 199_999)), ((429_000, 430_000), (0, 3, 500, 999))):
        cut = slice(seg[0], seg[1])
        small = [x[cut][:1000] if seg[0] == 0 else x[cut] for x in (q, k, v)]
        for h in (0, 39):
            qs, ks, vs = (x.cpu() for x in (q[cut], k[cut], v[cut]))
            ro, rl = owin.rows(qs, ks, vs, (0, seg[1] - seg[0]), h, rows, 200, 3)
            at = [seg[0] + i for i in rows]
            assert np.abs(f64(o[at, h]) - ro).max() <= 2e-2 and np.abs(f64(lse[h, at]) - rl).max() <= 2e-3
        del small
    # the last segment whole: its gradients are its own
    cut = slice(429_000, 430_000)
    qs, ks, vs = (x[cut].contiguous() for x in (q, k, v))
    one = torch.tensor([0, 1000], dtype=torch.int32, device="cuda")
    o1, l1 = vcs.attn_fwd_window(qs, ks, vs, one, 1000, 200, 3)
    assert torch.equal(o1, o[cut]) and torch.equal(l1, lse[:, cut])
    got = vcs.attn_bwd_window(qs, ks, vs, o1, l1, qs, one, 1000, 200, 3)
    for a, b in zip(got, (dq, dk, dv)):
        assert (a.double() - b[cut].double()).norm() <= 1e-3 * a.double().norm()


def test_on_streams_and_in_graphs():
    vcs = _vcs()
    lens = [700, 300, 2500]
    q, k, v, do = workloads.draw_dense(2, sum(lens), 4, 2, 64, device="cuda")
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    o, lse = vcs.attn_fwd_window(q, k, v, cu, 2500, 130, 4)
    want = vcs.attn_bwd_window(q, k, v, o, lse, do, cu, 2500, 130, 4)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for s in sides:  # two calls at once
        with torch.cuda.stream(s):
            torch.cuda._sleep(10_000_000)
        a = vcs.attn_fwd_window(q, k, v, cu, 2500, 130, 4, stream=s, check=False)
        got.append((*a, *vcs.attn_bwd_window(q, k, v, *a, do, cu, 2500, 130, 4, stream=s.cuda_stream, check=False)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = vcs.attn_fwd_window(q, k, v, cu, 2500, 130, 4, check=False)
        got.append((*a, *vcs.attn_bwd_window(q, k, v, *a, do, cu, 2500, 130, 4, check=False)))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for x in got:
        assert torch.equal(x[0], o) and torch.equal(x[1], lse) and all(torch.equal(p, w) for p, w in zip(x[3:], want[1:]))
        assert (x[2].double() - want[0].double()).norm() <= 1e-3 * want[0].double().norm()


@pytest.mark.parametrize("hq,hkv,d,window,sinks,inter", [(4, 2, 64, 100, 4, False), (3, 1, 128, 300, 0, True)])
def test_rotated_windowed_step_against_the_oracle(hq, hkv, d, window, sinks, inter):
    # layout, positions, rotated rows, windowed attention, and the gradients' way back to the trajectory rows
    vcs = _vcs()
    rng = np.random.default_rng(d)
    cu = np.array([0, 4, 9], np.int32)
    grid = np.stack([np.ones(9, int), rng.integers(4, 9, 9), rng.integers(5, 12, 9)], 1).astype(np.int32)
    img, txt = grid.prod(1).astype(np.int32), rng.integers(0, 30, 9).astype(np.int32)
    t = int(img.sum() + txt.sum())
    cud, imgd, txtd = steps_to_device(cu, img, txt)
    lay = vcs.build_segments(cud, imgd, txtd, 2, 1)
    sections = (d // 8, 3 * d // 16, 3 * d // 16)
    rope = vcs.rope_plan(d, sections, 1e4, interleaved=inter)
    pos = vcs.stream_positions(lay["cu_seqlens"], lay["tok_src_step"], imgd, txtd, torch.from_numpy(grid).cuda())
    off, tok = vcs.gather_inverse(lay["tok_gather"], t)
    qt, kt, vt, _ = workloads.draw_dense(d, t, hq, hkv, d, device="cuda")
    q, k, v = vcs.gather_rope(qt, kt, vt, lay["tok_gather"], pos, rope)
    args = (lay["cu_seqlens"], lay["max_seqlen"], window, sinks)
    o, lse = vcs.attn_fwd_window(q, k, v, *args)
    do = workloads.draw_dense(d + 1, lay["num_tokens"], hq, hkv, d, device="cuda")[0]
    grads = vcs.attn_bwd_window(q, k, v, o, lse, do, *args)
    back = vcs.gather_rope_bwd(*grads, pos, off, tok, rope)
    # the oracle from the trajectory rows on, nothing rounded on the way
    cus, src, gat = (lay[x].cpu().numpy() for x in ("cu_seqlens", "tok_src_step", "tok_gather"))
    po = orope.positions(cus, src, img, txt, grid)
    inv, axis = orope.frequencies(d, sections, 1e4)
    qr, kr = (orope.rotate(f64(x)[gat], po, inv, axis, inter) for x in (qt, kt))
    r = owin.attn(qr, kr, f64(vt)[gat], cus, window, sinks, f64(do))
    want = [orope.scatter(orope.rotate(r[x], po, inv, axis, inter, back=True) if x != "dv" else r[x], gat, t)
            for x in ("dq", "dk", "dv")]
    # rounding q and k to bf16 on the way moves a score by up to 2^-7 |q||k| scale: a few 1e-2 at these sizes
    assert np.linalg.norm(f64(o) - r["o"]) <= 1e-2 * np.linalg.norm(r["o"])
    for a, b in zip(back, want):
        assert np.linalg.norm(f64(a) - b) <= 1.5e-2 * np.linalg.norm(b)
