"""What the microscaled kernels may and may not promise to the compiler, from their source."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_12396_amd", "csrc")


def code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"/\*.*?\*/", "", re.sub(r"//[^\n]*", "", text), flags=re.S)


def test_shared_memory_is_read_where_it_was_written():
    """Direct loads fill shared memory through one pointer, and after the workgroup has met it is read through another: a pointer that promised
    to be the only one to its memory would let the compiler read before the meeting."""
    for name in ("nz_mx4.hip", "nz_mx4.hpp", "nz_mx4_product.hip"):
        assert not re.search(r"\b(__)?restrict(__)?\b|\bnoalias\b", code(name)), name


def test_every_meeting_is_fenced():
    """What was read, written and loaded before stays before, has ended when the workgroup meets, and nothing after is read early."""
    text = re.sub(r"\s+", " ", code("nz_mx4_product.hip"))
    meeting = ('__builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup"); __builtin_amdgcn_s_waitcnt(0x0070); __builtin_amdgcn_s_barrier(); '
               '__builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");')
    assert text.count("__builtin_amdgcn_s_barrier()") == text.count(meeting) > 0
