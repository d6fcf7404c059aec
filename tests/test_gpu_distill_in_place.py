"""GPU: distillation whose gradient goes over the logits, against the same call with the gradient apart."""
import pytest
import torch

from tests.test_gpu_distill import check, draw

pytestmark = pytest.mark.gpu


def _vcs():
    from paper_2607_11185_gb300 import vcs
    return vcs


@pytest.mark.parametrize("dtype,vocab,rows,top", [(torch.bfloat16, 131_072, 300, 64), (torch.bfloat16, 65_537, 900, 8),
                                                  (torch.float32, 99_991, 200, 300), (torch.float32, 160_000, 7, 1024),
                                                  (torch.bfloat16, 40_000, 3, 33), (torch.float32, 17_001, 1200, 20)])
def test_over_the_logits_beside_other_traffic(dtype, vocab, rows, top):
    # rows that a cluster shares, their entries spread over all its CTAs; another stream keeps the memory busy
    vcs = _vcs()
    z, ids, t, w = draw(vocab, rows, vocab, top, dtype)
    want = vcs.distill_topk(z, ids, t, w, temperature=1.1)
    a, b = (torch.zeros(1 << 27, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(12):
        over = z.clone()
        with torch.cuda.stream(side):
            for _ in range(3):
                b.copy_(a)
        got = vcs.distill_topk(over, ids, t, w, temperature=1.1, out=over, check=False)
        for x, y in zip(got, want):
            assert torch.equal(x, y)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_cluster_whose_shares_hold_no_finite_logit(dtype):
    # a masked vocabulary: the entries and all finite logits in one CTA's share
    z, ids, t, w = draw(1, 4, 131_072, 24, dtype)
    z[:2, :120_000] = -float("inf")
    z[2:, 9000:] = -float("inf")
    ids[:2] = torch.arange(125_000, 125_024, dtype=torch.int32)
    ids[2:] = torch.arange(24, dtype=torch.int32)
    check(z, ids, t, w)
    check(z, ids, t, w, out=z)
