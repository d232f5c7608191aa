"""Page bookkeeping at lengths near the largest int: refused, and nothing changes (a growth past it once wrapped round)."""
import subprocess
import sys

CODE = """
import ctypes as C
from paper_2606_31580_amd import laser as L
h = C.c_void_p()
L._call("laser_pages_create", 8, 16, 2, 4, C.byref(h))
lib = L.lib()
n = C.c_int()
for length in (2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16, 65):
    assert lib.laser_pages_add_seq(h, 0, length) == L.ERR_INVALID_ARG, length
L._call("laser_pages_add_seq", h, 0, 15)
for more in (2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16, 2 ** 31 - 31, 50):
    assert lib.laser_pages_append(h, 0, more) == L.ERR_INVALID_ARG, more
    L._call("laser_pages_seq_len", h, 0, C.byref(n))
    assert n.value == 15
L._call("laser_pages_append", h, 0, 49)
L._call("laser_pages_num_free", h, C.byref(n))
assert n.value == 4
print("ok")
"""


def test_lengths_near_the_largest_int():
    # (in a process of its own: an exception that passes a C entry ends it)
    r = subprocess.run([sys.executable, "-c", CODE], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr[-500:]
