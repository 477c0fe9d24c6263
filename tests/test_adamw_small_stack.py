"""CPU test of halo_adamw called by a thread that has a small stack, as the threads of some runtimes and pools have: lists of any length are
checked there, and refused with a status.  In a process of its own, which a stack that overflows would end."""
import os
import subprocess
import sys

import pytest

from paper_2501_02625_amd import _build

PROGRAM = r"""
import ctypes, sys, threading
from paper_2501_02625_amd import binding
lib = binding.load_library()
count = int(sys.argv[1])
def tensor(k):
    base = 0x10000000 * (k + 1)
    return binding.AdamwTensor(1000, base, base + 0x100000, base + 0x200000, base + 0x300000, None, base + 0x400000, base + 0x500000)
tensors = (binding.AdamwTensor * (count + 1))(*[tensor(k) for k in range(count)], tensor(0))         # the last one is the first one again
d = binding.AdamwDesc(0, 0, 8, 0, 1, 1e-3, 0.9, 0.95, 1e-8, 0.1, 1.0, 1, 2, None, None, None)
said = []
threading.stack_size(128 * 1024)
t = threading.Thread(target=lambda: said.append(lib.halo_adamw(ctypes.byref(d), tensors, count + 1, None)))
t.start()
t.join()
print(said[0])
"""


@pytest.mark.parametrize("count", [1, 47, 1023])
def test_tensors_given_twice(count):
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    done = subprocess.run([sys.executable, "-c", PROGRAM, str(count)], capture_output=True, text=True, cwd=_build.ROOT)
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])
    assert done.stdout.split() == ["1"]                                  # HALO_EINVAL
