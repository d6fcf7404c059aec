"""How blocks leave early, read from the kernels' source (CPU only).

Once a call has given up on a wait, blocks that start later stand down.  The status word may be set between two threads'
reads: one thread's read decides for the block, as warps that went on without those that allocate tensor memory, or
a warp without some of its lanes, would fault.
"""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_11185_gb300", "csrc")
FILES = sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def source(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def stand_downs(src):
    """Statements that leave on a time-out in the status word: (all, those of a thread by itself)."""
    found = [m.group() for m in re.finditer(r"[^;{}]*VCS_ERR_DEVICE_TIMEOUT[^;{}]*\breturn\b[^;{}]*;", src)
             if "return \"" not in m.group()]
    one = [x for x in found if not re.search(r"__syncthreads_or\(threadIdx\.x == 0 && ", x)]
    return found, one


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_one_thread_decides_whether_a_block_stands_down(path):
    found, one = stand_downs(source(path))
    assert one == []
    if os.path.basename(path) in ("attn_fwd.cu", "attn_bwd.cu", "attn_window.cu", "linear.cu"):
        assert found


def test_the_reader_sees_a_thread_by_itself():
    src = """{ const int st = *status; if (st == VCS_ERR_DEVICE_TIMEOUT) return; set_status(s, VCS_ERR_DEVICE_TIMEOUT);
      if (__syncthreads_or(threadIdx.x == 0 && *status == VCS_ERR_DEVICE_TIMEOUT)) return; }"""
    found, one = stand_downs(src)
    assert len(found) == 2 and one == [" if (st == VCS_ERR_DEVICE_TIMEOUT) return;"]
