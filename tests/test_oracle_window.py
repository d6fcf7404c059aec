"""Pins of the windowed attention oracle (CPU): the causal oracle, a library special case, differences."""
import numpy as np
import pytest
import torch

from oracle import attention as oatt
from oracle import window as owin


def draw(seed, n, hq, hkv, d):
    rng = np.random.default_rng(seed)
    return [rng.normal(size=(n, h, d)) for h in (hq, hkv, hkv, hq)]


CU = [0, 1, 1, 20, 57]


def test_a_wide_window_is_causal():
    q, k, v, do = draw(0, 57, 4, 2, 8)
    o, lse = oatt.attn_fwd(q, k, v, CU)
    dq, dk, dv = oatt.attn_bwd(q, k, v, do, CU)
    for window, sinks in ((37, 0), (10 ** 9, 3), (1, 37), (5, 10 ** 9)):
        r = owin.attn(q, k, v, CU, window, sinks, do)
        for name, want in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            assert np.allclose(r[name], want, atol=1e-12)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 2), (3, 0), (4, 1), (16, 5), (2, 30)])
def test_against_a_library_with_the_mask_spelled_out(window, sinks):
    q, k, v, _ = draw(1, 57, 4, 2, 8)
    r = owin.attn(q, k, v, CU, window, sinks)
    for b, e in zip(CU[:-1], CU[1:]):
        mask = torch.tensor([[j <= i and (j > i - window or j < sinks) for j in range(e - b)] for i in range(e - b)],
                            dtype=torch.bool).reshape(e - b, e - b)
        for h in range(4 if e > b else 0):
            x = [torch.tensor(t[b:e, i]) for t, i in ((q, h), (k, h // 2), (v, h // 2))]
            want = torch.nn.functional.scaled_dot_product_attention(*(t[None] for t in x), attn_mask=mask)[0]
            assert np.allclose(r["o"][b:e, h], want.numpy(), atol=1e-12)
            s = (x[0] @ x[1].T / 8 ** 0.5).masked_fill(~mask, -np.inf)
            assert np.allclose(r["lse"][h, b:e], torch.logsumexp(s, 1).numpy(), atol=1e-12)


def test_only_itself():
    q, k, v, do = draw(2, 57, 2, 1, 8)
    r = owin.attn(q, k, v, CU, 1, 0, do)
    assert np.allclose(r["o"], np.repeat(v, 2, 1)) and np.allclose(r["dv"], do.sum(1, keepdims=True))
    assert not np.abs(r["dq"]).max() > 1e-12 and not np.abs(r["dk"]).max() > 1e-12


def test_gradients_against_differences():
    q, k, v, do = draw(3, 12, 2, 1, 4)
    cu, window, sinks = [0, 5, 12], 3, 2
    r = owin.attn(q, k, v, cu, window, sinks, do)
    f = lambda: (owin.attn(q, k, v, cu, window, sinks)["o"] * do).sum()  # noqa: E731
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        for i in np.ndindex(*x.shape):
            keep = x[i]
            x[i] = keep + 1e-5
            up = f()
            x[i] = keep - 1e-5
            down = f()
            x[i] = keep
            assert abs((up - down) / 2e-5 - r[name][i]) < 1e-7


def test_chosen_rows():
    q, k, v, _ = draw(4, 57, 4, 2, 8)
    r = owin.attn(q, k, v, CU, 6, 3)
    for h in range(4):
        o, lse = owin.rows(q, k, v, (20, 57), h, [0, 1, 5, 6, 9, 36], 6, 3)
        at = [20 + i for i in (0, 1, 5, 6, 9, 36)]
        assert np.allclose(o, r["o"][at, h]) and np.allclose(lse, r["lse"][h, at])
