"""What attention over pages does on the host where there is no GPU: importing the binding, and the message of a launch that fails."""
import os
import subprocess
import sys

from paper_2604_18348_amd import binding as B
from tests.test_block_refusals import lib, params  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_binding_imports_with_a_torch_without_gpu_support():
    """Such a torch has no _cuda_* names in torch._C."""
    code = ("import torch\n"
            "for n in [n for n in dir(torch._C) if n.startswith('_cuda_')]: delattr(torch._C, n)\n"
            "from paper_2604_18348_amd import binding\n"
            "assert binding.BlockParams(B=1, Hq=1, Hkv=1, d=64).blocks == 1\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


SHIM = """
static int error;                                  // as the runtime keeps it: asking for it clears it
extern "C" int __hipPushCallConfiguration(...) { return 0; }
extern "C" int __hipPopCallConfiguration(...) { return 0; }
extern "C" int hipLaunchKernel(...) { return error = 98; }
extern "C" int hipGetLastError() { int e = error; error = 0; return e; }
extern "C" int hipPeekAtLastError() { return error; }
extern "C" const char* hipGetErrorString(int e) { return e == 98 ? "the launch was refused" : e ? "another error" : "no error"; }
"""

CALLS = """
import ctypes, sys
ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)       # ahead of the runtime in the search for names
lib = ctypes.CDLL(sys.argv[2])
text, one, size = ctypes.create_string_buffer(256), ctypes.c_void_p(256), ctypes.c_size_t(1 << 30)
for line in sys.stdin:
    name, blob, *args = line.split()
    args = [size if a == "size" else one if a == "1" else int(a[1:]) if a[0] == "i" else ctypes.c_void_p(0) for a in args]
    rc = getattr(lib, "adacluster_" + name)(*([] if blob == "-" else [bytes.fromhex(blob)]), *args)
    lib.adacluster_last_error(text, 256)
    print(name, rc, text.value.decode())
"""


def test_a_failed_launch_says_why(lib, tmp_path):  # noqa: F811
    """A runtime whose launches fail: every call returns ADACLUSTER_E_INTERNAL with the error of the launch, and leaves none behind."""
    (tmp_path / "shim.cpp").write_text(SHIM)
    shim = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-o", shim, str(tmp_path / "shim.cpp")], check=True)
    paged, packed = params(), params(num_pages=0, k_rows=9)
    calls = [("cache_append", paged, "1 1 1 1 1 1 1 0 0 1 0"), ("cache_read", paged, "1 1 1 1 1 0 0 1 1 0"), ("block_boxes", packed, "1 1 1 0"),
             ("block_select", paged, "1 1 0 1 1 1 1 1 1 size 0"), ("block_attn", paged, "1 1 1 1 0 0 0 1 1 0 1 1 1 size 0"),
             ("block_attn_backward", packed, "1 1 1 1 1 1 1 1 0 1 1 1 1 size 0"), ("block_attn_backward", packed, "1 1 1 1 1 1 1 1 1 1 1 1 1 size 0"),
             ("quest_scores", None, "i1 i32 i32 i64 i%d i0 i0 1 1 1 1 0" % B.F32)]
    lines = "".join("%s %s %s\n" % (name, "-" if c is None else bytes(c).hex(), args) for name, c, args in calls)
    r = subprocess.run([sys.executable, "-c", CALLS, shim, B.LIB_PATH], input=lines, capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    assert r.stdout.splitlines() == ["%s -6 HIP launch failed: the launch was refused" % name for name, _, _ in calls]
