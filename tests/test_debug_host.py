"""RRS_DEBUG's checks copy to host memory: where there is none the call fails with a status, and no C++
exception leaves the library (no GPU needed)."""
import subprocess
import sys

import paper_2409_20361_amd as rrs

# The check of float16 inputs, by its name in the library: no input that a call accepts is too
# large for the host everywhere.
CHECK = """
import ctypes
f = ctypes.CDLL({path!r})._ZN3rrs22debug_check_finite_f16EPKvmPKcPv
f.restype = ctypes.c_int32
f.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_char_p, ctypes.c_void_p]
for count in (1 << 62, 1 << 56):
    print(f(0x10000, count, b"X", None), flush=True)
"""


def test_no_host_memory():
    r = subprocess.run([sys.executable, "-c", CHECK.format(path=rrs.lib_path())],
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-300:]
    assert r.stdout.split() == ["-8", "-8"]
