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


@pytest.mark.parametrize("dtype,vocab,rows", [(torch.bfloat16, 20_011, 700), (torch.bfloat16, 131_072, 500), (torch.float32, 99_991, 160),
                                              (torch.bfloat16, 50_000, 3), (torch.float32, 1_000_003, 5)])
def test_two_calls_at_once_and_graphs_of_rows_in_clusters(dtype, vocab, rows):
    vcs = _vcs()
    a, b = (draw(seed, rows, vocab, 40, dtype) for seed in (1, 2))
    want = [vcs.distill_topk(*x, temperature=0.9) for x in (a, b)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = [vcs.distill_topk(*a, temperature=0.9, check=False), vcs.distill_topk(*b, temperature=0.9, stream=side, check=False),
               vcs.distill_topk(*a, temperature=0.9, check=False)]
        torch.cuda.synchronize()
        for x, y in zip(got, (want[0], want[1], want[0])):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
    graphs = []
    for x in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = vcs.distill_topk(*x, temperature=0.9, check=False)
        graphs.append((graph, out))
    for p, q in zip(a, b):       # each replay with the other's inputs
        p_old = p.clone()
        p.copy_(q)
        q.copy_(p_old)
    for _, out in graphs:
        for y in out:
            y.fill_(9.0)
    for i in (0, 1, 1, 0):
        graphs[i][0].replay()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.current_stream())
        graphs[1][0].replay()
    torch.cuda.synchronize()
    for (_, out), y in zip(graphs, want[::-1]):
        assert all(torch.equal(p, q) for p, q in zip(out, y))
