"""GPU: calls of linear attention that its documentation allows, on pointers, sizes and layouts of other kinds."""
import pytest
import torch

from tests.test_gpu_linear import decays

pytestmark = pytest.mark.gpu


def _vcs():
    from paper_2607_11185_gb300 import vcs
    return vcs


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 1, 2, 3])
def test_no_tokens_with_the_decays_of_one_layer(d, at):
    # a row of [layers, 2]: aligned to 4 bytes as fp32 is, not to 16; the states go through
    vcs = _vcs()
    g = decays(*[-0.01 * i for i in range(12)])[at:at + 2]
    q, k = (torch.zeros(0, h, d, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    state = torch.randn(3, 2, d, d, device="cuda")
    o, out = vcs.linear_attn_fwd(q, k, k, g, cu, state=state, with_state=True)
    assert o.shape == (0, 4, d) and torch.equal(out, state)
    assert not vcs.linear_attn_fwd(q, k, k, g, cu, with_state=True)[1].any()
    for x in vcs.linear_attn_bwd(q, k, k, q, g, cu):
        assert x.numel() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("decay", [-0.3, -1.1, -0.01])
def test_states_hold_the_bits_of_a_weighted_key(d, decay):
    # A segment whose first token alone has a key: its state is one product, e^(decay (n - 1)) k v.  Errors of it, relative:
    #   the weight's argument  |decay| (n - 1) (2^-25 + 2^-24 of log2's factor and product, 2^-24 of their product)
    #   exp2f                  2^-22 (2 ulp)
    #   times the key          2^-24, of which three bf16 terms leave 2^-27
    #   three accumulations    2 2^-23 (the tensor pipe may cut off)
    # in all below 2^-20 + |decay| (n - 1) 2^-22.  Two terms would leave 2^-18, and 2^-19 on average.
    vcs = _vcs()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    lens = list(range(2, 17)) + [100, 129, 300]
    cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    g = decays(decay, decay * 0.77)
    k = torch.zeros(sum(lens), 2, d, device="cuda")
    k[cu[:-1].long()] = torch.randn(len(lens), 2, d, generator=gen, device="cuda")
    k = k.to(torch.bfloat16)
    v = torch.randn(sum(lens), 2, d, generator=gen, device="cuda").to(torch.bfloat16)
    q = torch.zeros(sum(lens), 2, d, dtype=torch.bfloat16, device="cuda")
    state = vcs.linear_attn_fwd(q, k, v, g, cu, with_state=True)[1].double()
    first = cu[:-1].long()
    gap = torch.tensor(lens, device="cuda").double() - 1
    want = torch.exp(g.double()[None] * gap[:, None])[..., None, None] * k[first].double()[..., None] * v[first].double()[:, :, None]
    bound = (2.0 ** -20 + g.double().abs()[None] * gap[:, None] * 2.0 ** -22)[..., None, None] * want.abs() + 2.0 ** -126
    over = (state - want).abs() - bound
    assert over.max() <= 0, ((state - want).abs() / want.abs().clamp(min=1e-30)).max()


def test_states_of_short_segments_in_norm():
    # the terms as above, added up: their errors are of either sign, their sizes above the sum's by no more than 10 here
    vcs = _vcs()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    lens = [3, 16, 40, 128, 7]
    cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    g = decays(-0.3, -0.02)
    q, k, v = (torch.randn(sum(lens), 2, 128, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    state = vcs.linear_attn_fwd(q, k, v, g, cu, with_state=True)[1].double()
    for s, (b, n) in enumerate(zip(cu.tolist(), lens)):
        w = torch.exp(g.double()[None] * torch.arange(n - 1, -1, -1, device="cuda").double()[:, None])
        want = torch.einsum("jha,jhb->hab", k[b:b + n].double() * w[..., None], v[b:b + n].double())
        assert (state[s] - want).norm() <= 2.0 ** -20 * want.norm(), s


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (6, 2)])
def test_tensors_aligned_to_16_bytes_only(d, hq, hkv):
    # rows behind a segment's last whole chunk are stored 32 bytes at a time, or 16 and 16
    vcs = _vcs()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    lens = [1, 127, 130, 300, 2300]
    n, cu = sum(lens), torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    g = decays(-0.02, -1.3)
    q, do = (torch.randn(n, hq, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))

    def off(x, elements):      # a copy 16 bytes behind a boundary of 32
        room = torch.full((x.numel() + 2 * elements,), 3.0, dtype=x.dtype, device="cuda")
        y = room[elements:elements + x.numel()].view(x.shape)
        assert y.data_ptr() % 32 == 16
        y.copy_(x)
        return room, y

    state = torch.randn(len(lens), hkv, d, d, generator=gen, device="cuda")
    want = (*vcs.linear_attn_fwd(q, k, v, g, cu, state=state, with_state=True), *vcs.linear_attn_bwd(q, k, v, do, g, cu))
    (_, q2), (_, k2), (_, v2), (_, d2), (_, s2) = off(q, 8), off(k, 8), off(v, 8), off(do, 8), off(state, 4)
    ro, o = off(q, 8)
    rs, out = off(state, 4)
    grads = [off(x, 8) for x in (q, k, v)]
    nb = max(f(len(lens), n, hq, hkv, d) for f in (vcs.vcs_linear_attn_fwd_workspace_size, vcs.vcs_linear_attn_bwd_workspace_size))
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    args = (cu, len(lens), n, hq, hkv, d, 0.0)
    assert vcs.vcs_linear_attn_fwd(q2, k2, v2, g, *args, s2, out, o, ws, nb) == 0
    assert int(ws[:4].view(torch.int32)) == 0
    assert vcs.vcs_linear_attn_bwd(q2, k2, v2, d2, g, *args, *(y for _, y in grads), ws, nb) == 0
    assert int(ws[:4].view(torch.int32)) == 0
    for x, y in zip((o, out, *(y for _, y in grads)), want):
        assert torch.equal(x, y)
    for room, pad in ((ro, 8), (rs, 4), *((r, 8) for r, _ in grads)):
        assert (room[:pad] == 3).all() and (room[-pad:] == 3).all()
