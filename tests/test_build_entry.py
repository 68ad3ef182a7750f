"""build() in a process that has the package loaded: every binding takes the new library and the
others' new records."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import ctypes, os, sys
import __graft_entry__ as entry
import paper_2608_23253_amd as E
from paper_2608_23253_amd import _lib, _serve, _step
before = [m._LIB for m in (_lib, _serve, _step)]
# (the build itself is not what is looked at)
os.makedirs(os.path.join(sys.argv[1], "paper_2608_23253_amd"))
with open(os.path.join(sys.argv[1], "paper_2608_23253_amd", "build.py"), "w") as f:
    f.write("def build(verbose=False):\\n    return 'nothing'\\n")
entry.ROOT = sys.argv[1]
entry.build()
assert _serve._LIB is _lib._LIB and _step._LIB is _lib._LIB
assert all(m._LIB is not b for m, b in zip((_lib, _serve, _step), before))
plan = E.rotary_plan(64)
# a call reaches the library's own checks: no shape
for f, n in ((_serve._LIB.e2s_rotate_positions, 6), (_step._LIB.e2s_norm_rotate, 8)):
    assert f(None, ctypes.byref(plan), *[None] * n) == _lib.ERR_NULL_POINTER
print("fine")
"""


def test_a_build_beside_the_loaded_package(tmp_path):
    run = subprocess.run([sys.executable, "-c", PROGRAM, str(tmp_path)], cwd=ROOT,
                         capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("fine"), run.stderr
