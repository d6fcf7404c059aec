"""max_seqlen is a bound on the segments' lengths: a loose one, up to INT32_MAX, gives what the longest segment gives.

The order of dq's atomic additions varies from run to run, so it is compared by norm (fp32 sums of some thousand terms,
rounded to bf16: far below 1e-3); so are the windowed dk and dv, whose sinks' sums may be parted otherwise.  The
gathered gradients are atomic sums throughout.  Everything else is equal bit for bit.  A bound that a segment passes is
reported, also one of 0.
"""
import numpy as np
import pytest
import torch

from paper_2607_11185_gb300 import workloads
from tests.gpu_cases import cu_from_lengths

pytestmark = pytest.mark.gpu
LENS = [300, 1000, 1, 0, 129]


def close(a, b):
    return (a.double() - b.double()).norm() <= 1e-3 * b.double().norm()


@pytest.mark.parametrize("bound", [0, 1, 999])
def test_bounds_that_are_too_small_are_reported(bound):
    from paper_2607_11185_gb300 import vcs
    n = sum(LENS)
    q, k, v, do = workloads.draw_dense(3, n, 2, 1, 64, device="cuda")
    cu = torch.from_numpy(cu_from_lengths(LENS)).cuda()
    gat = torch.arange(n, dtype=torch.int32, device="cuda")
    o, lse = vcs.attn_fwd(q, k, v, cu, max(LENS))
    for call in (lambda: vcs.attn_fwd(q, k, v, cu, bound), lambda: vcs.attn_bwd(q, k, v, o, lse, do, cu, bound),
                 lambda: vcs.attn_fwd_gathered(q, k, v, gat, cu, bound),
                 lambda: vcs.attn_bwd_gathered(q, k, v, gat, o, lse, do, cu, bound),
                 lambda: vcs.attn_fwd_window(q, k, v, cu, bound, 200, 5),
                 lambda: vcs.attn_bwd_window(q, k, v, o, lse, do, cu, bound, 200, 5)):
        with pytest.raises(vcs.VcsError) as e:
            call()
        assert e.value.status == 6


@pytest.mark.parametrize("bound", [sum(LENS), 5000, 2 ** 31 - 128, 2 ** 31 - 1])
@pytest.mark.parametrize("d", [64, 128])
def test_loose_bounds(d, bound):
    from paper_2607_11185_gb300 import vcs
    n = sum(LENS)
    q, k, v, do = workloads.draw_dense(d, n, 4, 2, d, device="cuda")
    cu = torch.from_numpy(cu_from_lengths(LENS)).cuda()
    gat = torch.from_numpy(np.random.default_rng(1).permutation(n).astype(np.int32)).cuda()

    def causal(mx):
        o, lse = vcs.attn_fwd(q, k, v, cu, mx)
        return (o, lse, *vcs.attn_bwd(q, k, v, o, lse, do, cu, mx))

    def gathered(mx):
        o, lse = vcs.attn_fwd_gathered(q, k, v, gat, cu, mx)
        return (o, lse, *vcs.attn_bwd_gathered(q, k, v, gat, o, lse, do, cu, mx))

    def windowed(mx, window=200, sinks=5):
        o, lse = vcs.attn_fwd_window(q, k, v, cu, mx, window, sinks)
        return (o, lse, *vcs.attn_bwd_window(q, k, v, o, lse, do, cu, mx, window, sinks))

    for f, exact in ((causal, (0, 1, 3, 4)), (gathered, (0, 1)), (windowed, (0, 1)),
                     (lambda mx: windowed(mx, 2 ** 31 - 1, 0), (0, 1, 3, 4))):
        want = f(max(LENS))
        for i, (x, y) in enumerate(zip(f(bound), want)):
            assert torch.equal(x, y) if i in exact else close(x, y), (bound, i)
