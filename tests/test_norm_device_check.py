"""Every norm, residual and checkpoint call refuses a device that is not a whole 256-CU chip, before anything is launched (CPU).

A child process puts its own hipGetDevice and hipDeviceGetAttribute, which report a device of 128 compute units, in front of the
runtime's and calls the library."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PARTITION = """
int hipGetDevice(int* device) { *device = 0; return 0; }
int hipDeviceGetAttribute(int* value, int attribute, int device) { (void)attribute; (void)device; *value = 128; return 0; }
"""

# arguments that pass every other check
CALLS = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from tests.test_norm_library_abi import ALL, call
import paper_2407_15892_amd as mst
lib = mst.load_norm_library()
print(*(call(lib, name) for name in ALL))
"""


def test_a_partitioned_device_is_refused(tmp_path):
    import paper_2407_15892_amd as mst
    if not os.path.exists(mst.norm_binding.NORM_LIB_PATH):
        from paper_2407_15892_amd.build import build
        build()
    compiler = shutil.which("gcc") or shutil.which("cc")
    if compiler is None:
        pytest.skip("no C compiler")
    source, fake = tmp_path / "partition.c", tmp_path / "partition.so"
    source.write_text(PARTITION)
    subprocess.run([compiler, "-shared", "-fPIC", "-o", str(fake), str(source)], check=True)
    out = subprocess.run([sys.executable, "-c", CALLS, str(fake), ROOT], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    assert out.stdout.split()[-9:] == ["-7"] * 9
