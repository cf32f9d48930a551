"""What the library and its binding remember between calls: ctypes lets several threads into them at once, first calls included."""
import glob
import os
import re
import threading

from paper_2602_06183_b200 import binding, build

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


def test_the_library_is_handed_out_only_when_its_signatures_are_set(monkeypatch):
    """Without its signature a function takes a device address as a 32-bit integer. A thread that asks while another one loads the library
    gets it complete (the fake holds the loading thread up in the middle of the signatures)."""
    real, half, go_on, got = binding.C.CDLL, threading.Event(), threading.Event(), []

    class Fake:
        def __init__(self, path):
            self.lib, self.n = real(path), 0

        def __getattr__(self, name):
            self.n += 1
            if self.n == 5:
                half.set()
                assert go_on.wait(20)
            return getattr(self.lib, name)
    build.build()
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding.C, "CDLL", Fake)
    first = threading.Thread(target=binding.lib)
    first.start()
    assert half.wait(20)
    monkeypatch.setattr(binding.C, "CDLL", real)
    second = threading.Thread(target=lambda: got.append(binding.lib().sf_check_status.argtypes))
    second.start()
    second.join(1.0)                                        # (it may wait for the first, or load for itself)
    go_on.set()
    first.join(20)
    second.join(20)
    assert got == [binding._SIGNATURES["sf_check_status"][1]]
