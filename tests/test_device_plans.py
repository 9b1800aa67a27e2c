"""Plans and workspaces are those of the current device (no GPU): the library is loaded beside a stand-in for the two calls that ask for it."""
import os
import subprocess
import sys

from paper_2605_20104_amd import build

STAND_IN = """
static int device = 0;
void set_device(int d) { device = d; }
int hipGetDevice(int* d) { if (device < 0) return 100; *d = device; return 0; }
int hipDeviceGetAttribute(int* value, int attribute, int d) { (void)attribute; *value = d == 0 ? 256 : 64; return 0; }
"""
PROGRAM = """
import ctypes, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
mx, whole = lib.graft_tree_attn_mx_workspace_bytes, lib.graft_tree_attn_workspace_bytes
mx.restype = whole.restype = ctypes.c_size_t
for device in (0, 1, 0, 70, -1, 1):
    stand_in.set_device(device)
    print(mx(8, 1, 8, 2, 128, 4096), whole(8, 1, 8, 2, 128, 4096, 1))
"""


def test_workspaces_follow_the_current_device(tmp_path):
    (tmp_path / "stand_in.c").write_text(STAND_IN)
    lib = str(tmp_path / "stand_in.so")
    subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", lib, str(tmp_path / "stand_in.c")], check=True)
    out = subprocess.run([sys.executable, "-c", PROGRAM, lib, build.LIB], check=True, stdout=subprocess.PIPE, text=True).stdout
    mx, whole = zip(*[[int(x) for x in line.split()] for line in out.splitlines()])
    assert mx[0] == 8 * 8 * 32 * (128 + 2) * 4              # two workgroups a compute unit, 16 heads of sequences
    assert mx[1] == 8 * 8 * 8 * (128 + 2) * 4
    assert mx == (mx[0], mx[1], mx[0], mx[1], mx[0], mx[1])                 # (no device: as with 256)
    assert whole == (whole[0], whole[1], whole[0], whole[1], whole[0], whole[1])
    assert whole[0] != whole[1]
