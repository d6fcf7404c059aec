"""Linear attention and distillation on the host (CPU only): calls that would read or write what they must not."""
import pytest

from tests.test_linear_host import bwd, distill, far, fwd, step


@pytest.fixture(scope="module")
def vcs():
    from paper_2607_11185_gb300 import vcs as v
    return v


def test_outputs_over_decays_and_bounds(vcs):
    row = 10 * 64 * 2                       # a key/value row tensor of 10 tokens; the queries' twice that
    for kw in (dict(o=far(3)), dict(o=far(3) - 2 * row + 16), dict(g=far(5) + 2 * row - 4), dict(so=far(3)),
               dict(o=far(4)), dict(o=far(4) - 2 * row + 16), dict(cu=far(5) + 2 * row - 8), dict(so=far(4)),
               dict(so=far(9), g=far(9) + 64 * 64 * 4 - 4)):
        assert fwd(vcs, **kw) == 1, kw
    for x, size in (("dq", 2 * row), ("dk", row), ("dv", row)):
        at = dict(dq=far(5), dk=far(7), dv=far(8))[x]
        for kw in (dict(g=at), dict(g=at + size - 4), dict(cu=at), dict(cu=at + size - 8), dict(cu=at - 4)):
            assert bwd(vcs, **kw) == 1, (x, kw)
    for kw in (dict(so=far(3)), dict(o=far(3)), dict(g=far(5) + 2 * row - 4), dict(g=far(4) + 10 * 64 * 64 * 4 - 4)):
        assert step(vcs, **kw) == 1, kw


def test_scalars_that_are_not_aligned_to_themselves(vcs):
    for f in (fwd, bwd, step):
        for off in (1, 2, 3):
            assert f(vcs, g=far(3) + off) == 1
    for f in (fwd, bwd):
        for off in (1, 2, 3):
            assert f(vcs, cu=far(4) + off) == 1
    assert step(vcs, w=far(7) + 2) == 1


def test_a_view_of_no_tokens_overlaps_nothing(vcs):
    # its address lies in another buffer's span: the refusal that comes next shows that the spans passed
    assert fwd(vcs, nt=0, q=None, k=None, v=None, si=far(9), so=far(10), o=far(9) + 64, ws=None) == 8
    assert fwd(vcs, nt=0, q=None, k=None, v=None, si=far(9), so=far(10), o=far(10) + 64, ws=None) == 8


def test_the_gradient_s_stride_without_a_gradient(vcs):
    # not looked at: the refusal that comes last is the workspace's
    for ldg in (-1, 0, 99, 1 << 62, (1 << 63) - 1):
        assert distill(vcs, g=None, ldg=ldg, ws=None) == 8


def test_temperatures_without_a_finite_inverse(vcs):
    for temp in (1e-45, 1e-40, 4e-39):
        assert distill(vcs, temp=temp) == 1
    for temp in (1e-38, 1e-30, 3e38):
        assert distill(vcs, temp=temp, ws=None) == 8
