"""GPU: linear attention and distillation as an update uses them together, each part against its oracle."""
import numpy as np
import pytest
import torch

from oracle import distill as odis
from oracle import linear as olin
from paper_2607_11185_gb300 import workloads
from tests.gpu_cases import cu_from_lengths
from tests.test_gpu_distill import HALF
from tests.test_gpu_linear import decays, f64, near

pytestmark = pytest.mark.gpu

LENS, HQ, HKV, D, VOCAB, TOP = [300, 1, 2200, 77, 129], 6, 2, 64, 1003, 16


def draw(seed):
    from paper_2607_11185_gb300 import vcs
    n = sum(LENS)
    q, k, v, _ = workloads.draw_dense(seed, n, HQ, HKV, D, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    mask = (torch.rand(n, generator=gen, device="cuda") < 0.1).to(torch.uint8)
    mask[-1] = 1
    head = (torch.randn(HQ * D, VOCAB, generator=gen, device="cuda") * 0.05).to(torch.bfloat16)
    rows = vcs.compact_trainable(mask)
    ids = torch.randint(0, VOCAB, (n, TOP), generator=gen, device="cuda", dtype=torch.int32)
    teacher = torch.randn(n, TOP, generator=gen, device="cuda") * 2
    weights = torch.full((rows.numel(),), 1.0 / rows.numel(), device="cuda")
    return q, k, v, head, rows, ids, teacher, weights


def update(q, k, v, head, rows, ids, teacher, weights, g, cu, check=True):
    """Outputs, logits of the trained tokens, their loss and gradient, and the gradients of q, k and v."""
    from paper_2607_11185_gb300 import vcs
    o, _ = vcs.linear_attn_fwd(q, k, v, g, cu, check=check)
    logits = o.view(len(o), -1)[rows.long()] @ head
    z = logits.clone()
    loss, kl, dz = vcs.distill_topk(logits, ids, teacher, weights, rows, 1.5, out=logits, check=check)   # in place
    do = torch.zeros_like(o)
    do.view(len(o), -1)[rows.long()] = dz @ head.T
    return o, z, loss, kl, dz, do, *vcs.linear_attn_bwd(q, k, v, do, g, cu, check=check)


def test_an_update():
    g, cu = decays(-0.004, -1.5), cu_from_lengths(LENS)
    cud = torch.from_numpy(cu).cuda()
    x = draw(0)
    q, k, v, head, rows, ids, teacher, weights = x
    o, z, loss, kl, dz, do, dq, dk, dv = update(*x, g, cud)
    r = olin.attn(q, k, v, g, cu)
    near(f64(o), r["o"], r["o_abs"], "o")
    lw, kw, gw = odis.distill(f64(z), ids.cpu().numpy(), f64(teacher), f64(weights), rows.cpu().numpy(), 1.5)
    size = np.abs(f64(teacher)).max() + np.abs(f64(z)).max()
    ek = 2.0 ** -17 + 2.0 ** -21 * size / 1.5          # the bounds of distillation's own tests, at their largest
    assert (np.abs(f64(kl) - kw) <= ek + 2.0 ** -24 * np.abs(kw)).all()
    assert abs(float(loss) - lw) <= ek + 2.0 ** -24 * abs(lw)
    far = 2.0 ** -16 + 2.0 ** -22 * max(88.0, 2 * np.abs(f64(z)).max() / 1.5)
    bound = f64(weights)[:, None] / 1.5 * far * 2 + HALF[dz.dtype] * np.abs(gw) + 2.0 ** -125
    assert (np.abs(f64(dz) - gw) <= bound).all()
    r = olin.grads(q, k, v, do, g, cu)
    for got, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        near(f64(got), r[name], r[name + "_abs"], name)


def test_captured_updates_on_new_inputs():
    g, cu = decays(-0.004, -1.5), torch.from_numpy(cu_from_lengths(LENS)).cuda()
    x = draw(0)
    update(*x, g, cu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = update(*x, g, cu, check=False)
    rows = x[4]
    for seed in (1, 2):
        new = draw(seed)
        for a, b in zip(x[:4] + x[5:7], new[:4] + new[5:7]):    # the trained tokens stay, their number is the graph's
            a.copy_(b)
        want = [y.clone() for y in update(*x, g, cu)]
        for y in out:
            y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
    assert rows.numel() > 100
