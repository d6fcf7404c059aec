"""GPU parity of linear attention against the fp64 oracle.

Elementwise bounds, from the roundings (u = 2^-8, half a step of bf16).  An output is a sum of terms
lam^(i-j) q_ia k_ja v_je, each with two roundings to bf16 at most: between the tokens of a chunk the weighted value (the
gradients of keys and values: the weighted query) and the product that multiplies it; through the state the weighted
value or key, and the state that the query reads.  The output itself is rounded once:
  |error| <= (2 u + u^2 + 2^-15) sum |terms| + u |o|
where 2^-15 holds the fp32 additions (2^-24 each; up to a chunk's 128 and a chunk's states one after another), the
decays' own rounding (a weight e^-x is off by x 2^-23, at most 0.4 2^-23 of 1) and their products from chunk to chunk.
States carry no bf16 rounding but a weighted key in three terms, which hold its 24 bits:
  |error| <= 2^-14 sum |terms|
The gradients are sums of the same kind, over their own terms.
"""
import numpy as np
import pytest
import torch

from oracle import linear as olin
from paper_2607_11185_gb300 import workloads
from tests.gpu_cases import cu_from_lengths

pytestmark = pytest.mark.gpu
U, FP, ST = 2.0 ** -8, 2.0 ** -15, 2.0 ** -14


def _vcs():
    from paper_2607_11185_gb300 import vcs
    return vcs


def f64(x):
    return x.double().cpu().numpy()


def within(got, want, bound, name):
    over = np.abs(got - want) - bound - 1e-30
    assert np.isfinite(got).all(), name
    assert over.size == 0 or over.max() <= 0, (name, int((over > 0).sum()), over.max(),
                                               np.unravel_index(over.argmax(), over.shape))


def near(got, want, size, name):
    within(got, want, (2 * U + U * U + FP) * size + U * np.abs(want), name)
    far = np.linalg.norm(got - want)
    assert far <= 6e-3 * np.linalg.norm(want) + U * U * np.linalg.norm(size), (name, far, np.linalg.norm(want))


def decays(*g):
    return torch.tensor(g, dtype=torch.float32, device="cuda")


def check(q, k, v, do, g, lens, scale=0.0, state=None):
    vcs = _vcs()
    cu = cu_from_lengths(lens)
    cud = torch.from_numpy(cu).cuda()
    o, end = vcs.linear_attn_fwd(q, k, v, g, cud, scale, state, with_state=True)
    plain, none = vcs.linear_attn_fwd(q, k, v, g, cud, scale, state)
    # of a segment that several CTAs share the state between them comes from keys in three terms or, without states as
    # results, in one: both within the bound
    assert none is None and (torch.equal(plain, o) or max(lens) > 2048)
    r = olin.attn(q, k, v, g, cu, state, scale)
    near(f64(o), r["o"], r["o_abs"], "o")
    near(f64(plain), r["o"], r["o_abs"], "o without states")
    within(f64(end), r["state"], ST * r["state_abs"], "state")
    got = vcs.linear_attn_bwd(q, k, v, do, g, cud, scale)
    r = olin.grads(q, k, v, do, g, cu, scale)
    for x, name in zip(got, ("dq", "dk", "dv")):
        near(f64(x), r[name], r[name + "_abs"], name)


LENS = [1, 2, 130, 0, 127, 128, 129, 257, 0, 385, 640]


def draw(seed, lens, hq, hkv, d):
    return workloads.draw_dense(seed, sum(lens), hq, hkv, d, device="cuda")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -0.01, -0.09, -0.7, -6.0, -90.0, -1e30])
def test_decays(d, decay):
    check(*draw(int(-decay * 1000) % 97, LENS, 3, 1, d), decays(decay), LENS)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (2, 2), (4, 2), (5, 1), (7, 1), (8, 4), (16, 2), (3, 3)])
def test_heads(d, hq, hkv):
    lens = [300, 129, 700, 64]
    g = decays(*[-(2.0 ** (-8 * (i + 1) / hkv)) for i in range(hkv)])
    check(*draw(hq * 10 + hkv, lens, hq, hkv, d), g, lens)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [1, 2, 127, 128, 129, 255, 256, 257, 383, 384, 385, 513])
def test_lengths(d, length):
    check(*draw(length, [length], 2, 1, d), decays(-0.02), [length])


@pytest.mark.parametrize("d,scale", [(64, 0.5), (128, 1e-3), (64, 30.0), (128, -1.0)])
def test_scales(d, scale):
    check(*draw(3, [400, 200], 4, 2, d), decays(-0.1, -0.003), [400, 200], scale)


@pytest.mark.parametrize("d", [64, 128])
def test_states(d):
    lens = [0, 1, 200, 128, 0, 300]
    q, k, v, do = draw(5, lens, 4, 2, d)
    gen = torch.Generator(device="cuda").manual_seed(1)
    state = torch.randn(len(lens), 2, d, d, generator=gen, device="cuda") * 20
    check(q, k, v, do, decays(-0.05, 0.0), lens, 0.0, state)
    vcs = _vcs()
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")   # no tokens at all: the states go through
    o, end = vcs.linear_attn_fwd(q[:0], k[:0], v[:0], decays(-0.05, 0.0), cu, state=state[:3].contiguous(), with_state=True)
    assert o.shape == (0, 4, d) and torch.equal(end, state[:3])
    o, end = vcs.linear_attn_fwd(q[:0], k[:0], v[:0], decays(-0.05, 0.0), cu, with_state=True)
    assert not end.any()
    assert vcs.linear_attn_fwd(q[:0], k[:0], v[:0], decays(-0.05, 0.0), cu[:1], with_state=True)[1].shape == (0, 2, d, d)
    assert [tuple(x.shape) for x in vcs.linear_attn_bwd(q[:0], k[:0], v[:0], do[:0], decays(-1.0, 0.0), cu)] == \
        [(0, 4, d), (0, 2, d), (0, 2, d)]


@pytest.mark.parametrize("d,hq,hkv", [(64, 14, 2), (128, 28, 4), (128, 40, 8), (64, 1, 1), (128, 16, 16), (64, 12, 1)])
@pytest.mark.parametrize("n", [1, 3, 100])
def test_step(d, hq, hkv, n):
    vcs = _vcs()
    q, k, v, _ = draw(n + hq, [n], hq, hkv, d)
    gen = torch.Generator(device="cuda").manual_seed(n)
    states = torch.randn(n, hkv, d, d, generator=gen, device="cuda")
    g = decays(*[-0.5 / (i + 1) for i in range(hkv - 1)], 0.0)
    before = states.clone()
    o = vcs.linear_attn_step(q, k, v, g, states)
    r = olin.attn(q, k, v, g, np.arange(n + 1), before)
    within(f64(o), r["o"], FP * r["o_abs"] + U * np.abs(r["o"]), "o")
    within(f64(states), r["state"], 2.0 ** -21 * r["state_abs"], "state")
    assert vcs.linear_attn_step(q[:0], k[:0], v[:0], g, states[:0]).shape == (0, hq, d)
    if n > 1:  # the first rows of a padded batch; the others' states stay
        part = before.clone()
        o2 = vcs.linear_attn_step(q[:n - 1], k[:n - 1], v[:n - 1], g, part[:n - 1])
        assert torch.equal(o2, o[:n - 1]) and torch.equal(part[:-1], states[:-1]) and torch.equal(part[-1], before[-1])


def test_prompt_then_tokens():
    # a prompt in two pieces and the rest token by token are the whole
    vcs = _vcs()
    hq, hkv, d, n = 6, 2, 128, 300
    q, k, v, _ = draw(8, [2 * n], hq, hkv, d)
    g = decays(-0.01, -0.2)
    cu = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    _, state = vcs.linear_attn_fwd(*(x[:150].contiguous() for x in (q, k, v)), g, cu(0, 150), with_state=True)
    a, state = vcs.linear_attn_fwd(*(x[150:n - 2].contiguous() for x in (q, k, v)), g, cu(0, n - 152), state=state,
                                   with_state=True)
    last = [vcs.linear_attn_step(*(x[t:t + 1].contiguous() for x in (q, k, v)), g, state) for t in (n - 2, n - 1)]
    r = olin.attn(q[:n], k[:n], v[:n], g, [0, n])
    near(f64(torch.cat([a, *last])), r["o"][150:], r["o_abs"][150:], "o")
    within(f64(state), r["state"], ST * r["state_abs"], "state")


def test_rows_of_no_segment_stay():
    vcs = _vcs()
    lens = [5, 200, 7, 130, 9]
    q, k, v, do = draw(4, lens, 4, 2, 64)
    cu = cu_from_lengths(lens)
    g = decays(-0.1, 0.0)
    part = torch.from_numpy(cu[1:-1].copy()).cuda()    # without the first and the last segment
    whole = torch.from_numpy(cu).cuda()
    names = ("linear_attn_fwd", "linear_attn_bwd")
    for name, extra in zip(names, ((), (do,))):
        want = getattr(vcs, name)(q, k, v, *extra, g, whole)
        nb = getattr(vcs, f"vcs_{name}_workspace_size")(3, len(q), 4, 2, 64)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        outs = [torch.full_like(x, 7.0) for x in want if x is not None]
        if extra:
            st = vcs.vcs_linear_attn_bwd(q, k, v, do, g, part, 3, len(q), 4, 2, 64, 0.0, *outs, ws, nb)
        else:
            st = vcs.vcs_linear_attn_fwd(q, k, v, g, part, 3, len(q), 4, 2, 64, 0.0, None, None, *outs, ws, nb)
        torch.cuda.synchronize()
        assert st == 0 and ws[:4].view(torch.int32).item() == 0
        for x, y in zip(outs, want):
            assert torch.equal(x[cu[1]:cu[-2]], y[cu[1]:cu[-2]])
            assert (x[:cu[1]] == 7).all() and (x[cu[-2]:] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("decay", [(-0.3, 0.0), (-4.0, -1.2)])
@pytest.mark.parametrize("hq", [2, 4, 6])
def test_segments_do_not_meet(d, decay, hq):
    # NaN and infinities in one segment are not seen by its neighbours, whose last tiles reach into it
    vcs = _vcs()
    lens = [100, 3, 150, 1, 70]
    q, k, v, do = draw(6, lens, hq, 2, d)
    cu, g = cu_from_lengths(lens), decays(*decay)
    cud = torch.from_numpy(cu).cuda()
    want = [*vcs.linear_attn_fwd(q, k, v, g, cud, with_state=True), *vcs.linear_attn_bwd(q, k, v, do, g, cud)]
    for bad, s in ((float("nan"), 1), (float("inf"), 3), (3e38, 1), (float("nan"), 2)):
        at = slice(cu[s], cu[s + 1])
        x = [t.clone() for t in (q, k, v, do)]
        for t in x:
            t[at] = bad
        got = [*vcs.linear_attn_fwd(*x[:3], g, cud, with_state=True), *vcs.linear_attn_bwd(*x, g, cud)]
        for i, (a, b) in enumerate(zip(got, want)):
            keep = torch.ones(len(a), dtype=torch.bool)
            keep[s if i == 1 else at] = False
            assert torch.equal(a[keep], b[keep]), (bad, s, i)


def test_the_same_bits_twice_and_on_another_stream():
    vcs = _vcs()
    lens = [3000, 700, 1, 5000]
    q, k, v, do = draw(9, lens, 10, 2, 128)
    g, cu = decays(-0.01, 0.0), torch.from_numpy(cu_from_lengths(lens)).cuda()
    calls = lambda **kw: [*vcs.linear_attn_fwd(q, k, v, g, cu, with_state=True, **kw),  # noqa: E731
                          *vcs.linear_attn_bwd(q, k, v, do, g, cu, **kw)]
    want = calls()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    both = [calls(check=False), calls(stream=side, check=False), calls(check=False)]
    torch.cuda.synchronize()
    for got in both:
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_graphs():
    # captured with its gradients and a step, replayed on new inputs; two graphs of their own workspaces
    vcs = _vcs()
    lens, g = [200, 5000, 3], decays(-0.02, 0.0)
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    x = draw(1, lens, 4, 2, 64)
    tok = [t[:3].contiguous() for t in x[:3]]
    states = torch.zeros(3, 2, 64, 64, device="cuda")

    def run():
        o, st = vcs.linear_attn_fwd(*x[:3], g, cu, with_state=True, check=False)
        states.copy_(st)
        return [o, *vcs.linear_attn_bwd(*x, g, cu, check=False), vcs.linear_attn_step(*tok, g, states, check=False)]

    run()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run())
        graphs.append(graph)
    for seed in (2, 3):
        for a, b in zip(x, draw(seed, lens, 4, 2, 64)):
            a.copy_(b)
        for graph, out in zip(graphs, outs):
            for y in out:
                y.fill_(9.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, run()):
                assert torch.equal(a, b)


def test_device_checks():
    vcs = _vcs()
    q, k, v, do = draw(2, [300], 2, 1, 64)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    good = i32(0, 100, 300)
    for cu in (i32(0, 200, 100), i32(0, 100, 301), i32(-1, 100, 300), i32(0, -5, 300), i32(0, 2 ** 31 - 1, 300),
               i32(300, 0)):
        for f in (lambda: vcs.linear_attn_fwd(q, k, v, decays(-1.0), cu), lambda: vcs.linear_attn_bwd(q, k, v, do, decays(-1.0), cu)):
            with pytest.raises(vcs.VcsError) as e:
                f()
            assert e.value.status == 6
    states = torch.ones(300, 1, 64, 64, device="cuda")
    for g in (1e-6, float("nan"), float("inf"), -float("inf")):
        for f in (lambda: vcs.linear_attn_fwd(q, k, v, decays(g), good),
                  lambda: vcs.linear_attn_bwd(q, k, v, do, decays(g), good),
                  lambda: vcs.linear_attn_step(q, k, v, decays(g), states)):
            with pytest.raises(vcs.VcsError) as e:
                f()
            assert e.value.status == 6
    assert (states == 1).all()
    # a bad segment leaves the others' results
    o, end = vcs.linear_attn_fwd(q, k, v, decays(-0.1), good, with_state=True)
    bad, end2 = vcs.linear_attn_fwd(q, k, v, decays(-0.1), i32(0, 100, 50, 500), with_state=True, check=False)
    torch.cuda.synchronize()
    assert torch.equal(bad[:100], o[:100]) and torch.equal(end2[0], end[0])


def test_refusals():
    vcs = _vcs()
    q, k, v, do = draw(2, [30], 4, 2, 64)
    g, cu, st = decays(-1.0, 0.0), torch.tensor([0, 30], dtype=torch.int32, device="cuda"), torch.zeros(1, 2, 64, 64, device="cuda")
    f, b, s = vcs.linear_attn_fwd, vcs.linear_attn_bwd, vcs.linear_attn_step
    for call in (lambda: f(q.float(), k, v, g, cu), lambda: f(q, k[:, :1], v, g, cu), lambda: f(q, k, v[:20], g, cu),
                 lambda: f(q.transpose(1, 2), k, v, g, cu), lambda: f(q, k, v, g[:1], cu), lambda: f(q, k, v, g.double(), cu),
                 lambda: f(q, k, v, g, cu.long()), lambda: f(q, k, v, g, cu, state=st[:0]), lambda: f(q, k, v, g, cu, state=st.double()),
                 lambda: f(q, k, v, g.cpu(), cu), lambda: f(q, k, v, g, cu.cpu()), lambda: f(q, k, v, g, cu, state=st.cpu()),
                 lambda: b(q, k, v, do[:10], g, cu), lambda: b(q, k, v, do.float(), g, cu), lambda: b(q, k, v, do.cpu(), g, cu),
                 lambda: s(q, k, v, g, st), lambda: s(q[:1], k[:1], v[:1], g, st.double()), lambda: s(q[:1], k[:1], v[:1], g, st.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(q[:, :3].contiguous(), k, v, g, cu), lambda: f(*(x[..., :32].contiguous() for x in (q, k, v)), g, cu),
                 lambda: s(*(x[:1, :, :32].contiguous() for x in (q, k, v)), g, torch.zeros(1, 2, 32, 32, device="cuda"))):
        with pytest.raises(vcs.VcsError) as e:
            call()
        assert e.value.status == 2


@pytest.mark.parametrize("d,hq,hkv,lens", [(64, 2, 1, [20_000, 9_000]), (128, 4, 2, [17_001, 128]), (128, 2, 2, [12_345])])
def test_long_segments(d, hq, hkv, lens):
    # sampled rows of segments of many chunks, the gradients' at the ends that gather most
    vcs = _vcs()
    q, k, v, do = draw(d + hq, lens, hq, hkv, d)
    cu = cu_from_lengths(lens)
    cud = torch.from_numpy(cu).cuda()
    g = decays(*([-0.0005, 0.0][:hkv]))
    o, end = vcs.linear_attn_fwd(q, k, v, g, cud, with_state=True)
    dq, dk, dv = vcs.linear_attn_bwd(q, k, v, do, g, cud)
    rng = np.random.default_rng(0)
    for b, e in zip(cu[:-1].tolist(), cu[1:].tolist()):
        rows = sorted({b, e - 1, *rng.integers(b, e, 12).tolist(), *[t for t in (b + 127, b + 128, e - 129) if b <= t < e]})
        for h in range(hkv):
            x = h * hq // hkv
            for t in rows:
                near(f64(o[t, x]), *olin.row(q, k, v, g[h], b, t, x, h), "o")
                near(f64(dq[t, x]), *olin.row(do, v, k, g[h], b, t, x, h), "dq")
                i = np.arange(t, e)
                w = np.exp(float(g[h]) * (i - t)) * d ** -0.5
                grp = range(x, x + hq // hkv)
                kt, vt, qs, ds = f64(k[t, h]), f64(v[t, h]), [f64(q[t:e, y]) for y in grp], [f64(do[t:e, y]) for y in grp]
                for got, row, a, c, name in ((dk[t, h], vt, ds, qs, "dk"), (dv[t, h], kt, qs, ds, "dv")):
                    want = sum((w * (y @ row)) @ z for y, z in zip(a, c))
                    size = sum((w * (np.abs(y) @ np.abs(row))) @ np.abs(z) for y, z in zip(a, c))
                    near(f64(got), want, size, name)
    for s, (b, e) in enumerate(zip(cu[:-1].tolist(), cu[1:].tolist())):
        for h in range(hkv):
            w = np.exp(float(g[h]) * np.arange(e - b - 1, -1, -1))[:, None]
            kk, vv = f64(k[b:e, h]), f64(v[b:e, h])
            within(f64(end[s, h]), (w * kk).T @ vv, ST * ((w * np.abs(kk)).T @ np.abs(vv)), "state")


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 4), (64, 12, 4), (128, 4, 4), (128, 8, 4), (128, 20, 4)])
def test_short_and_cut_segments_with_heads_of_all_paces(d, hq, hkv):
    # several pieces to a CTA, sequences over several of them, the exact powers beside the weighted tiles
    lens = [2600, 1, 130, 0, 64, 300, 128] + [17, 200] * 10 + [2177, 5]
    check(*draw(d + hq, lens, hq, hkv, d), decays(-0.0003, 0.0, -0.5, -5.0), lens)
    state = torch.randn(len(lens), hkv, d, d, device="cuda")
    vcs = _vcs()
    q, k, v, _ = draw(1, lens, hq, hkv, d)
    g, cu = decays(-3.0, -0.0003, -0.02, 0.0), cu_from_lengths(lens)
    o, end = vcs.linear_attn_fwd(q, k, v, g, torch.from_numpy(cu).cuda(), 0.0, state, with_state=True)
    r = olin.attn(q, k, v, g, cu, state)
    near(f64(o), r["o"], r["o_abs"], "o")
    within(f64(end), r["state"], ST * r["state_abs"], "state")


@pytest.mark.parametrize("d", [64, 128])
def test_the_lowest_decay(d):
    # nothing of the last token is left at the next
    lens, g = [1, 130, 2100], decays(-torch.finfo(torch.float32).max, 0.0)
    check(*draw(3, lens, 4, 2, d), g, lens)
    vcs = _vcs()
    q, k, v, _ = draw(4, [5], 4, 2, d)
    st = torch.randn(5, 2, d, d, device="cuda")
    want = k[:, 0, :, None].float() * v[:, 0, None, :].float()
    vcs.linear_attn_step(q, k, v, g, st)
    assert torch.equal(st[:, 0], want)


def test_rows_past_2_31_elements():
    lens, hq, hkv, d = [900] * 470 + [333], 40, 8, 128
    assert (sum(lens) - 333) * hq * d > 2 ** 31
    q, k, v, do = draw(5, lens, hq, hkv, d)
    vcs = _vcs()
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    g = decays(*([-0.01, 0.0, -2.0, -0.3] * 2))
    o, _ = vcs.linear_attn_fwd(q, k, v, g, cu)
    grads = vcs.linear_attn_bwd(q, k, v, do, g, cu)
    end = [x[-333:] for x in (q, k, v, do)]
    r = olin.attn(*end[:3], g, [0, 333])
    near(f64(o[-333:]), r["o"], r["o_abs"], "o")
    r = olin.grads(*end, g, [0, 333])
    for x, name in zip(grads, ("dq", "dk", "dv")):
        near(f64(x[-333:]), r[name], r[name + "_abs"], name)


def test_no_tokens_and_no_segments():
    vcs = _vcs()
    q, k, v, do = draw(6, [7], 4, 2, 64)
    none = [x[:0] for x in (q, k, v, do)]
    g, st = decays(-0.1, 0.0), torch.randn(3, 2, 64, 64, device="cuda")
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    o, end = vcs.linear_attn_fwd(*none[:3], g, cu, state=st, with_state=True)
    assert o.shape == (0, 4, 64) and torch.equal(end, st)
    o, end = vcs.linear_attn_fwd(*none[:3], g, cu, with_state=True)
    assert (end == 0).all()
    assert all(x.shape[0] == 0 for x in vcs.linear_attn_bwd(*none, g, cu))
    o, end = vcs.linear_attn_fwd(q, k, v, g, cu[:1], with_state=True)
    assert o.shape == q.shape and end.shape[0] == 0
    o, end = vcs.linear_attn_fwd(q, k, v, g, cu, state=st, with_state=True)   # segments without tokens among some
    assert torch.equal(end, st)
    assert vcs.linear_attn_step(*none[:3], g, st[:0]).shape == (0, 4, 64)


@pytest.mark.parametrize("d,hq,hkv,n", [(64, 1024, 1, 140), (128, 320, 320, 30), (64, 600, 300, 300), (128, 200, 1, 2100)])
def test_many_heads(d, hq, hkv, n):
    lens = [n // 2, n - n // 2] if n < 2000 else [n]
    q, k, v, do = draw(hq, lens, hq, hkv, d)
    g = decays(*np.linspace(-3, 0, hkv).tolist())
    vcs = _vcs()
    cu = cu_from_lengths(lens)
    cud = torch.from_numpy(cu).cuda()
    o, end = vcs.linear_attn_fwd(q, k, v, g, cud, with_state=True)
    grads = vcs.linear_attn_bwd(q, k, v, do, g, cud)
    for h in sorted({0, hkv // 2, hkv - 1}):    # a state's heads by themselves
        x = slice(h * hq // hkv, (h + 1) * hq // hkv)
        part = [q[:, x], k[:, h:h + 1], v[:, h:h + 1], do[:, x]]
        r = olin.attn(*part[:3], g[h:h + 1], cu)
        near(f64(o[:, x]), r["o"], r["o_abs"], "o")
        within(f64(end[:, h:h + 1]), r["state"], ST * r["state_abs"], "state")
        r = olin.grads(*part, g[h:h + 1], cu)
        for got, name, y in zip(grads, ("dq", "dk", "dv"), (x, slice(h, h + 1), slice(h, h + 1))):
            # (dk and dv of a group of hundreds: as many more additions, 2^-24 of the sum each)
            near(f64(got[:, y]), r[name], r[name + "_abs"], name)


def test_thousands_of_segments():
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 6, size=2600)]
    check(*draw(7, lens, 2, 1, 64), decays(-0.2), lens)


def test_states_past_2_31_elements():
    n, hkv, d = 16_600, 8, 128
    assert (n - 3) * hkv * d * d > 2 ** 31
    vcs = _vcs()
    q, k, v, _ = draw(8, [n], 8, hkv, d)
    st = torch.zeros(n, hkv, d, d, device="cuda")
    st[-2:] = torch.randn(2, hkv, d, d, device="cuda")
    before = st[-3:].clone()
    g = decays(*([-0.1, 0.0] * 4))
    o = vcs.linear_attn_step(q, k, v, g, st)
    want, end = olin.walk(q[-3:], k[-3:], v[-3:], g, [0, 1, 2, 3], state=before)
    # states: three roundings of 2^-24 of at most 30; outputs: half a step of bf16, and 128 additions of 2^-24 of a sum of
    # sizes below 14
    assert np.abs(f64(st[-3:]) - end).max() <= 1e-5
    assert np.abs(f64(o[-3:]) - want).max() <= U * np.abs(want).max() + 1e-4


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 8), (64, 8, 8), (128, 16, 8), (64, 24, 8)])
def test_many_runs_have_the_same_bits(d, hq, hkv):
    # heads of all paces over segments that CTAs share: a wait that is missing shows as a run in a hundred
    lens = [8000, 7875]
    q, k, v, do = draw(9, lens, hq, hkv, d)
    g = decays(-0.7, 0.0, -2.0, -0.69, -14.0, -1.7, -0.05, -3.0)
    cu = torch.from_numpy(cu_from_lengths(lens)).cuda()
    vcs = _vcs()

    def run():
        o, end = vcs.linear_attn_fwd(q, k, v, g, cu, with_state=True, check=False)
        return [o, end, vcs.linear_attn_fwd(q, k, v, g, cu, check=False)[0],
                *vcs.linear_attn_bwd(q, k, v, do, g, cu, check=False)]

    want = run()
    for _ in range(120):
        for x, y in zip(run(), want):
            assert torch.equal(x, y)
