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
