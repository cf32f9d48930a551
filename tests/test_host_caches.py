"""What the library and its binding remember between calls: ctypes lets several threads into them at once, first calls included."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_06183_b200", "csrc")
# of a thread of its own, atomic inside, or by contract of one thread (sf_trace_set)
ALLOWED = re.compile(r"thread_local|std::atomic|\bFewRoom \w+(\[64\])?;|g_trace_")


def test_remembered_values_are_atomic():
    variable = re.compile(r"^(?: +static (?!const\b|constexpr\b|__device__)|(?:thread_local |std::\S+ |const |unsigned |int |bool |cudaEvent_t\* )+g_)[^()\n]*[;{=][^\n]*$", re.M)
    seen = 0
    for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        for m in variable.finditer(open(p).read()):
            seen += 1
            assert ALLOWED.search(m.group(0)), (os.path.basename(p), m.group(0).strip())
    assert seen >= 15
