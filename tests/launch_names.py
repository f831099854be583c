"""Which kernels a call of the C ABI launches, without a GPU: HIP's own functions are replaced, in a process of its own,
by ones that launch nothing and note the names."""
import json
import subprocess
import sys
import textwrap

STUB = r"""
#include <stdio.h>
#include <string.h>
typedef struct { unsigned x, y, z; } dim3;
static const void *host[4096];
static const char *device[4096];
static int known;
static dim3 grid, block;
static size_t shared;
static void *queue;
static char log_[1 << 16];
void __hipRegisterFunction(void **m, const void *h, char *d, const char *name) {
    if (known < 4096) host[known] = h, device[known++] = name;
}
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t n, void *s) { grid = g, block = b, shared = n, queue = s; return 0; }
int __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *n, void **s) { *g = grid, *b = block, *n = shared, *s = queue; return 0; }
int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **args, size_t n, void *s) {
    for (int i = 0; i < known; ++i)
        if (host[i] == f) {
            const size_t at = strlen(log_);
            snprintf(log_ + at, sizeof log_ - at, "%s %u %u %u\n", device[i], g.x, g.y, b.x);
        }
    return 0;
}
int hipGetLastError(void) { return 0; }
int hipFuncSetAttribute(void) { return 0; }
const char *launches(void) { return log_; }
void forget(void) { log_[0] = 0; }
"""

CALLS = textwrap.dedent("""
    import ctypes, json, sys
    stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(sys.argv[2])
    stub.launches.restype = ctypes.c_char_p
    kinds = dict(p=ctypes.c_void_p, i=ctypes.c_int, l=ctypes.c_longlong, f=ctypes.c_float)
    out = []
    for name, args in json.load(sys.stdin):
        stub.forget()
        status = getattr(lib, name)(*(None if v is None else kinds[k](v) for k, v in args))
        out.append((status, [line.split() for line in stub.launches().decode().splitlines()]))
    print(json.dumps(out))
""")

FAR = 1 << 44   # apart: no tensor meets another


def launches(calls, library, folder):
    """[(status, [[mangled name, grid x, grid y, threads]])] of calls [(name, [(kind, value)])], kinds "pilf"."""
    (folder / "stub.c").write_text(STUB)
    (folder / "calls.py").write_text(CALLS)
    subprocess.run(["gcc", "-shared", "-fPIC", "-w", str(folder / "stub.c"), "-o", str(folder / "stub.so")], check=True)
    r = subprocess.run([sys.executable, str(folder / "calls.py"), str(folder / "stub.so"), library], input=json.dumps(calls),
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return [(s, [(n, int(x), int(y), int(t)) for n, x, y, t in ls]) for s, ls in json.loads(r.stdout)]


def window_call(B, H, Hk, Lq, Lk, D, frame=1, window=0, sinks=0, dtype=0):
    p = [("p", FAR * i) for i in range(1, 8)]
    p[3] = p[4] = ("p", None)
    sizes = (B, H, Hk, Lq, Lk, D, frame, window, sinks)
    return ("sdattn_window_forward", p + [("l", 1 << 40)] + [("i", n) for n in sizes] + [("f", 0.125), ("i", 1), ("i", 1), ("i", dtype), ("p", None)])


def cache_call(B, H, Hk, Lq, D, slots, frame=1, window=0, sinks=0, dtype=0):
    p = [("p", FAR * i) for i in range(1, 11)]
    sizes = (B, H, Hk, Lq, D, B * slots, slots, frame, window, sinks)
    return ("sdattn_cache_forward", p + [("l", 1 << 40)] + [("i", n) for n in sizes] + [("f", 0.125), ("i", 1), ("i", 1), ("i", dtype), ("p", None)])
