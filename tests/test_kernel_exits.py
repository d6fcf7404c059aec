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


def functions(src):
    """Bodies of the functions and kernels that stand at the file's outer levels, by their names."""
    out = {}
    for m in re.finditer(r"\n(?:template [^\n]*\n)?[a-z_][^;{}()]*?\b(\w+)\(", src):
        at = src.find("{", m.end())
        semi = src.find(";", m.end())
        if at < 0 or 0 <= semi < at:
            continue
        depth = 0
        for end in range(at, len(src)):
            depth += (src[end] == "{") - (src[end] == "}")
            if depth == 0:
                break
        out.setdefault(m.group(1), src[at:end])
    return out


def kernels_that_move_registers(src):
    out = []
    for m in re.finditer(r"__launch_bounds__\(.*?\)\s*\n?\s*(\w+)\(", src):
        at = src.index("{", src.index(")", m.end()))
        nxt = src.find("__global__", at)
        if "setmaxnreg_inc<" in src[at:nxt if nxt > 0 else len(src)]:
            out.append(m.group(1))
    return out


def launches(src):
    """Kernels that move registers, the functions that launch them, and whether these check the build's registers."""
    return [(k, f, "launch_regs_match(" in b) for k in kernels_that_move_registers(src) for f, b in functions(src).items()
            if re.search(r"\b%s<[^;{}()]*>\s*<<<" % k, b)]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_a_kernel_that_moves_registers_is_launched_with_what_it_counts_on(path):
    # a warpgroup that asks for more than the block was launched with would wait without a limit
    found = launches(source(path))
    assert {k for k, *_ in found} == set(kernels_that_move_registers(source(path)))
    assert [x for x in found if not x[2]] == []


def test_the_readers_of_launches_find_them():
    moving = {k for p in FILES for k in kernels_that_move_registers(source(p))}
    assert {"attn_fwd_kernel", "attn_window_kernel", "bwd_main", "linear_states", "linear_out", "linear_back"} <= moving
    src = """
__global__ void __launch_bounds__(512, 1)
    kernel(int a) { setmaxnreg_inc<C::R>(); }

template <int D>
cudaError_t go(int x) { kernel<D><<<1, 512>>>(x); return 0; }
template <int D>
cudaError_t checked(int x) { launch_regs_match(fn, 128, &c, &ok); kernel<D><<<1, 512>>>(x); return 0; }
"""
    assert launches(src) == [("kernel", "go", False), ("kernel", "checked", True)]


def left_open(src):
    """Kernels that may end with loads or MMAs under way where a wait has run out: (kernel, barriers of loads, MMAs end)."""
    out = []
    for k in kernels_that_move_registers(src):
        at = re.search(r"__launch_bounds__\(.*?\)\s*\n?\s*%s\(" % k, src).start()
        nxt = src.find("__global__", at)
        b = src[at:nxt if nxt > 0 else len(src)]
        end = re.search(r"__syncthreads\(\);\s*if \(gave_up\(\)\) \{(.*)\n  \}\n  if \(warp == \d\) \{", b, re.S)
        end = end.group(1) if end else ""
        filled = set(re.findall(r"mbar_arrive_expect_tx\(&bars->(\w+)", b))
        filled |= set(re.findall(r"load\(\w+::\w+, bars->(\w+),", b))           # through a function of the kernel
        waited = set(re.findall(r"finish_loads\(bars->(\w+)", end))
        out.append((k, filled - waited, "finish_mmas(" in end))
    return [x for x in out if x[1] or not x[2]]


def test_what_a_block_has_under_way_ends_before_it():
    # where a wait has run out nobody else waits for it, and it would write into the next block's shared memory
    with open(os.path.join(CSRC, "linear.cu")) as f:
        assert left_open(f.read()) == []
