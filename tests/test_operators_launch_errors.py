"""What a launch that HIP refuses comes back as: HIP's error, from every entry point of the
adapters, the norms with rotation and the selected blocks.  HIP's own functions are replaced by
ones that launch nothing (in a process of its own), so no GPU."""
import os
import subprocess
import sys
import textwrap

import pytest

from paper_2304_11267_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID_CONFIGURATION = 9

STUB = r"""
static int launches;
int hipLaunchKernel(void) { ++launches; return %d; }
int hipGetLastError(void) { return launches ? %d : 0; }
int hipFuncSetAttribute(void) { return 0; }
int __hipPushCallConfiguration(void) { return 0; }
int __hipPopCallConfiguration(void) { return 0; }
int launched(void) { const int n = launches; launches = 0; return n; }
""" % (INVALID_CONFIGURATION, INVALID_CONFIGURATION)

CALLS = textwrap.dedent("""
    import ctypes, sys
    stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(sys.argv[2])
    p = [ctypes.c_void_p(0x10000000 * i) for i in range(1, 10)]
    f = ctypes.c_float
    big = ctypes.c_longlong(1 << 27)
    x, w, bias, down, up, ids, scales, y, ws = p
    for name, args in (
            ("sdattn_linear_adapters", (x, w, bias, down, up, ids, scales, y, ws, big, 4, 70, 320, 640, 20, 3, 8, 0, 1, 0)),
            ("sdattn_linear_adapters", (x, w, bias, down, up, ids, scales, y, ws, big, 4, 1, 320, 640, 64, 3, 8, 0, 0, 1)),
            ("sdattn_norm_rotate", (x, w, None, None, None, None, up, y, 2, 8, 100, 40, 0, None, 1, 1, f(1e-6), 0, 0, 1, 1)),
            ("sdattn_block_means", (x, y, 2, 8, 1000, 40, 0)),
            ("sdattn_select_blocks", (x, w, y, 2, 8, 1000, 70, 40, 64, 9, 0)),
            ("sdattn_select_blocks", (x, w, y, 8, 8, 1000, 70, 40, 64, 9, 0)),
            ("sdattn_sparse_forward", (x, w, bias, down, y, 2, 8, 1000, 900, 64, 64, f(0.125), 0)),
            ("sdattn_sparse_forward", (x, w, bias, down, y, 2, 8, 1, 900, 64, 64, f(0.125), 1))):
        status = getattr(lib, name)(*args, None)
        print(name, status, lib.sdattn_last_hip_error(), stub.launched(), flush=True)
""")


def test_a_refused_launch_is_an_error_of_hip(tmp_path):
    if not os.path.exists(binding.library_path()):
        pytest.skip("libsdattn.so not built")
    (tmp_path / "stub.c").write_text(STUB)
    (tmp_path / "calls.py").write_text(CALLS)
    subprocess.run(["gcc", "-shared", "-fPIC", "-w", str(tmp_path / "stub.c"), "-o", str(tmp_path / "stub.so")], check=True)
    r = subprocess.run([sys.executable, str(tmp_path / "calls.py"), str(tmp_path / "stub.so"), binding.library_path()],
                       cwd=ROOT, capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    lines = [line.split() for line in r.stdout.splitlines()]
    assert len(lines) == 8
    for name, status, error, launched in lines:
        assert int(launched) == 1, name   # the first refused launch ends the call
        assert (int(status), int(error)) == (binding.STATUS_HIP, INVALID_CONFIGURATION), name
