"""GPU parity of distillation from a teacher's top logits against the fp64 oracle.

Bounds.  ln sum exp is off by at most 2^-17: the exponentials by 2^-21 of themselves and 2^-23 of their argument's
size (whose terms e^-x x stay below 0.4), the fp32 sums by 2^-24 an addition in trees (what a thread's chain rounds off
is kept beside it).  A list's log
p_j and z_j / T are off by 2^-22 of their size.  So
  kl       2^-17 + 2^-21 max (|t_j| + |z_j|) / T
  dlogits  |w| / T ((2^-16 + 2^-22 x) q + (2^-16 + 2^-22 88) p) + half a step of its type of itself
where x = (max z - z) / T is the exponential's argument: the difference, its factor and their product are rounded once
each (2^-24) and T itself to fp32 (2^-25 of what the oracle is given), 3.5 2^-24 x < 2^-22 x in all, which is no small
part of 2^-16 where q is; p's arguments likewise, below 88 where p is not flushed.  An exponential below 2^-126 is
flushed to 0, which |w| / T multiplies, and so is a gradient.
  loss     sum |w| (error of kl) + 2^-24 of itself
"""
import math

import numpy as np
import pytest
import torch

from oracle import distill as odis

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _vcs():
    from paper_2607_11185_gb300 import vcs
    return vcs


def draw(seed, rows, vocab, top, dtype=torch.float32, lists=None, pad=0, twice=False):
    rng = np.random.default_rng(seed)
    lists = rows if lists is None else lists
    z = torch.from_numpy(rng.normal(size=(rows, vocab + pad)) * 3).to(dtype).cuda()[:, :vocab]
    ids = rng.integers(0, vocab, size=(lists, top)) if twice else np.array(
        [rng.permutation(vocab)[:top] if top <= vocab else rng.integers(0, vocab, top) for _ in range(lists)]).reshape(lists, top)
    t = rng.normal(size=(lists, top)) * 2 + 5
    w = rng.normal(size=rows)
    return (z, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(t).float().cuda(),
            torch.from_numpy(w).float().cuda())


def check(z, ids, t, w, rows=None, temp=1.0, **kw):
    vcs = _vcs()
    n, vocab = z.shape
    zn = z.double().cpu().numpy()
    only = vcs.distill_topk(z, ids, t, w, rows, temp, with_grad=False)
    loss, kl, g = vcs.distill_topk(z, ids, t, w, rows, temp, **kw)
    assert only[2] is None
    assert loss.dtype == kl.dtype == torch.float32 and g.dtype == z.dtype and g.shape == z.shape
    idn, tn, wn = ids.cpu().numpy(), t.double().cpu().numpy(), w.double().cpu().numpy()
    rn = None if rows is None else rows.cpu().numpy()
    lw, kw_, gw = odis.distill(zn, idn, tn, wn, rn, temp)
    at = np.arange(n) if rn is None else rn
    here = (idn[at] >= 0) & np.isfinite(tn[at])
    size = np.where(here, np.abs(np.where(here, tn[at], 0)) + np.abs(np.take_along_axis(zn, np.maximum(idn[at], 0), 1)), 0)
    ek = 2.0 ** -17 + 2.0 ** -21 * size.max(1, initial=0) / temp
    for ls, x in ((loss, kl), only[:2]):   # with the gradient, and without, where the sums may be in another order
        dk = np.abs(x.double().cpu().numpy() - kw_)
        assert (dk <= ek + 2.0 ** -24 * np.abs(kw_)).all(), (dk.max(), ek.max())
        assert abs(float(ls) - lw) <= (np.abs(wn) * ek).sum() + 2.0 ** -24 * abs(lw)
    c = np.abs(wn)[:, None] / temp
    live = (wn != 0) & here.any(1)
    lz = zn / temp - (zn / temp).max(1, keepdims=True)
    q = np.exp(lz) / np.exp(lz).sum(1, keepdims=True) * live[:, None]
    p = np.abs(q - np.divide(gw, (wn / temp)[:, None], out=np.zeros_like(gw), where=live[:, None]))
    far = np.minimum(-lz, 1e3)
    bound = c * ((2.0 ** -16 + 2.0 ** -22 * far) * q + (2.0 ** -16 + 2.0 ** -22 * 88) * p) \
        + HALF[z.dtype] * np.abs(gw) + 2.0 ** -126 * (1 + c)
    dg = np.abs(g.double().cpu().numpy() - gw)
    assert (dg <= bound).all(), (dg.max(), np.unravel_index((dg - bound).argmax(), dg.shape))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 31, 100, 511, 1000, 1024, 1025, 4099, 8192, 20001])
def test_vocabularies(dtype, vocab):
    check(*draw(vocab, 5, vocab, min(vocab, 20), dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab,rows", [(50_001, 3), (131_072, 2), (160_000, 3), (299_999, 2), (1_000_003, 1)])
def test_large_vocabularies(dtype, vocab, rows):
    check(*draw(vocab, rows, vocab, 64, dtype), temp=1.3)


@pytest.mark.parametrize("top", [1, 2, 3, 31, 32, 33, 255, 511, 512, 513, 1023, 1024])
def test_lists(top):
    check(*draw(top, 4, 3000, top, torch.bfloat16))
    check(*draw(top, 3, 200, top, twice=True))


@pytest.mark.parametrize("temp", [1e-2, 0.5, 1.0, 2.0, 37.0, 1e4])
def test_temperatures(temp):
    check(*draw(3, 6, 1500, 30), temp=temp)


@pytest.mark.parametrize("rows", [1, 2, 3, 151, 152, 153, 700, 2500])
def test_rows(rows):
    check(*draw(rows, rows, 97, 6, torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [1, 3, 8, 61])
def test_rows_apart(dtype, pad):
    z, ids, t, w = draw(pad, 9, 1003, 12, dtype, pad=pad)
    check(z, ids, t, w)
    room = torch.full((9, 1003 + 2 * pad), 7.0, dtype=dtype, device="cuda")
    check(z, ids, t, w, out=room[:, pad:pad + 1003])
    assert (room[:, :pad] == 7).all() and (room[:, pad + 1003:] == 7).all()
    whole = torch.as_strided(z, (9, 1003 + pad), (1003 + pad, 1))
    behind = whole[:, 1003:].clone()
    check(z, ids, t, w, out=z)    # the gradient over the logits
    assert torch.equal(whole[:, 1003:], behind)


def test_lists_by_row():
    z, ids, t, w = draw(4, 40, 600, 9, lists=70)
    rows = torch.from_numpy(np.random.default_rng(2).integers(0, 70, 40).astype(np.int32)).cuda()
    check(z, ids, t, w, rows)
    check(z, ids, t, w)           # more lists than rows


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_absent_entries_and_idle_rows(dtype):
    z, ids, t, w = draw(5, 60, 900, 16, dtype)
    rng = np.random.default_rng(1)
    ids[torch.from_numpy(rng.random((60, 16)) < 0.4).cuda()] = -1
    t[torch.from_numpy(rng.random((60, 16)) < 0.1).cuda()] = -math.inf
    ids[7] = -1
    t[8] = -math.inf
    idle = torch.from_numpy(rng.random(60) < 0.3).cuda()
    w[idle] = 0.0
    w[7:9] = 1.0
    bare = z.clone()
    bare[idle] = math.nan         # not read
    vcs = _vcs()
    got = vcs.distill_topk(bare, ids, t, w)
    for a, b in zip(got, vcs.distill_topk(z, ids, t, w)):
        assert torch.equal(a, b)
    assert not got[2][idle].any() and not got[1][idle].any() and not got[2][7:9].any()
    check(z, ids, t, w)


def test_far_apart_logits():
    z, ids, t, w = draw(6, 4, 5000, 10)
    z[0] *= 1000
    z[1, :4000] = -math.inf       # a masked vocabulary
    ids[1] = torch.arange(4500, 4510)
    z[2] = 1e30
    t[3] *= 1e4
    check(z, ids, t, w, temp=0.7)


def test_infinities_and_nan():
    vcs = _vcs()
    z, ids, t, w = draw(7, 6, 700, 10)
    z[0, 5] = math.nan
    t[1, 3] = math.nan
    z[2] = -math.inf
    t[3, 2] = math.inf
    z[4, int(ids[4, 0])] = -math.inf   # the student excludes what the teacher has
    want = vcs.distill_topk(z[5:], ids[5:], t[5:], w[5:])
    loss, kl, g = vcs.distill_topk(z, ids, t, w)
    assert torch.isnan(kl[:4]).all() and torch.isposinf(kl[4]) and torch.isnan(loss).all() | torch.isinf(loss).all()
    assert torch.isnan(g[:4]).any(1).all() and torch.isfinite(g[4:]).all()
    assert torch.equal(kl[5:], want[1]) and torch.equal(g[5:], want[2])


def test_device_checks():
    vcs = _vcs()
    z, ids, t, w = draw(8, 5, 300, 7)
    for at, bad in (((2, 3), 300), ((0, 0), -2), ((4, 6), 2 ** 31 - 1), ((1, 1), -2 ** 31)):
        x = ids.clone()
        x[at] = bad
        with pytest.raises(vcs.VcsError) as e:
            vcs.distill_topk(z, x, t, w)
        assert e.value.status == 6
        y = ids.clone()
        y[at] = -1
        for a, b in zip(vcs.distill_topk(z, x, t, w, check=False), vcs.distill_topk(z, y, t, w)):
            assert torch.equal(a, b)
    for bad in (5, -1, 2 ** 31 - 1):
        rows = torch.arange(5, dtype=torch.int32, device="cuda")
        rows[3] = bad
        with pytest.raises(vcs.VcsError) as e:
            vcs.distill_topk(z, ids, t, w, rows)
        assert e.value.status == 6
        _, kl, g = vcs.distill_topk(z, ids, t, w, rows, check=False)
        assert kl[3] == 0 and not g[3].any() and (kl[:3] != 0).all()


def test_no_rows():
    vcs = _vcs()
    z, ids, t, w = draw(8, 5, 300, 7)
    loss, kl, g = vcs.distill_topk(z[:0], ids, t, w[:0])
    assert float(loss) == 0 and kl.shape == (0,) and g.shape == (0, 300)
    none = torch.zeros(5, dtype=torch.int32, device="cuda")
    with pytest.raises(vcs.VcsError) as e:       # no lists at all: every row's is outside
        vcs.distill_topk(z, ids[:0], t[:0], w, none)
    assert e.value.status == 6


def test_refusals():
    vcs = _vcs()
    z, ids, t, w = draw(8, 5, 300, 7)
    f, m = vcs.distill_topk, torch.zeros(5, dtype=torch.int32, device="cuda")
    for call in (lambda: f(z.half(), ids, t, w), lambda: f(z.double(), ids, t, w), lambda: f(z[0], ids, t, w),
                 lambda: f(z.T, ids, t, w), lambda: f(z[:1].expand(5, 300), ids, t, w), lambda: f(z, ids.long(), t, w),
                 lambda: f(z, ids, t.bfloat16(), w), lambda: f(z, ids, t[:, :6], w), lambda: f(z, ids, t, w[:4]),
                 lambda: f(z, ids, t, w.double()), lambda: f(z, ids, t, w, m[:4]), lambda: f(z, ids, t, w, m.long()),
                 lambda: f(z, ids, t, w, out=z[:4]), lambda: f(z, ids, t, w, out=z.bfloat16()),
                 lambda: f(z, ids, t, w, out=z, with_grad=False), lambda: f(z.cpu(), ids, t, w),
                 lambda: f(z, ids, t, w.cpu()), lambda: f(z, ids, t, w, out=z.cpu())):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(5, 1025, dtype=torch.int32, device="cuda")
    for call, code in ((lambda: f(z, ids[:4], t[:4], w), 1), (lambda: f(z, ids, t, w, temperature=0.0), 1),
                       (lambda: f(z, wide, wide.float(), w), 2), (lambda: f(z, ids[:, :0], t[:, :0], w), 1),
                       (lambda: f(z, ids, t, w, out=torch.as_strided(z, (5, 300), (300, 1), 0)[:, :]), 0)):
        if code:
            with pytest.raises(vcs.VcsError) as e:
                call()
            assert e.value.status == code
        else:
            call()


def test_the_same_bits_twice_two_calls_at_once_and_graphs():
    vcs = _vcs()
    z, ids, t, w = draw(9, 900, 2111, 24, torch.bfloat16)
    want = vcs.distill_topk(z, ids, t, w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [vcs.distill_topk(z, ids, t, w, check=False), vcs.distill_topk(z, ids, t, w, stream=side, check=False),
           vcs.distill_topk(z, ids, t, w, check=False)]
    torch.cuda.synchronize()
    for x in got:
        for a, b in zip(x, want):
            assert torch.equal(a, b)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(vcs.distill_topk(z, ids, t, w, check=False))
        graphs.append(graph)
    for seed in (1, 2):
        for a, b in zip((z, ids, t, w), draw(seed, 900, 2111, 24, torch.bfloat16)):
            a.copy_(b)
        want = vcs.distill_topk(z, ids, t, w)
        for graph, out in zip(graphs, outs):
            for y in out:
                y.fill_(9.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_rows_past_2_31_elements():
    # bf16 rows whose offsets do not fit 32 bits: the last rows against the same rows alone
    vcs = _vcs()
    rows, vocab = 17_000, 131_072
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda").normal_()
    ids = (torch.arange(rows * 8, device="cuda", dtype=torch.int32).view(rows, 8) * 7919) % vocab
    t = torch.randn(rows, 8, device="cuda")
    w = torch.ones(rows, device="cuda")
    tail = [x[-3:].clone() for x in (z, ids, t, w)]
    want = vcs.distill_topk(*tail)
    _, kl, g = vcs.distill_topk(z, ids, t, w, out=z)
    # (few rows are split over more of the chip, in another order of their sums: 2^-16 of both, a step of the rounding)
    assert ((kl[-3:] - want[1]).abs() <= 2.0 ** -16).all()
    assert ((g[-3:].double() - want[2].double()).abs() <= (2.0 ** -15 + 2.0 ** -7) * want[2].double().abs()).all()


@pytest.mark.parametrize("dtype,vocab,rows", [(torch.bfloat16, 131_072, 5), (torch.float32, 160_000, 3), (torch.bfloat16, 32_000, 200),
                                              (torch.bfloat16, 3001, 700), (torch.float32, 2_000_003, 1)])
def test_in_place_and_entries_twice_on_every_route(dtype, vocab, rows):
    # one CTA a row, clusters of them, blocks in turn, rows beyond a cluster; a list's ids from few, at both ends of the row
    vcs = _vcs()
    z, ids, t, w = draw(vocab, rows, vocab, 64, dtype)
    ids = torch.where(ids % 2 == 0, ids % 20, vocab - 1 - ids % 20).contiguous()
    check(z, ids, t, w, temp=0.7)
    loss, kl, want = vcs.distill_topk(z, ids, t, w, temperature=0.7)
    over = z.clone()
    again = vcs.distill_topk(over, ids, t, w, temperature=0.7, out=over)
    assert again[2] is over and torch.equal(over, want) and torch.equal(again[0], loss) and torch.equal(again[1], kl)


@pytest.mark.parametrize("rows", [304, 305, 1300])
def test_the_loss_alone_by_blocks_of_every_size(rows):
    z, ids, t, w = draw(rows, rows, 9001 if rows < 1000 else 40_007, 20, torch.bfloat16)
    check(z, ids, t, w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(1, 1_000_003), (2, 100_000), (1, 3_000_001), (320, 9000)])
@pytest.mark.parametrize("below", [0.0, 1.0, 3.3])
def test_rows_of_equal_logits(dtype, rows, vocab, below):
    # every addition of a chain rounds the same way
    z, ids, t, w = draw(1, rows, vocab, 16, dtype)
    z.fill_(-below)
    z[:, vocab // 3] = 0.0
    check(z, ids, t, w)
