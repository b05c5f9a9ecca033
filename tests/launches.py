"""Which kernels a call of the library launches, without a GPU: the few runtime functions that a launch needs are replaced by ones that keep a record, in a process
of their own."""
import json
import os
import subprocess
import sys

from paper_2501_07145_amd import binding

RUNTIME = r"""
#include <stddef.h>
#include <string.h>
typedef struct { unsigned x, y, z; } dim3;
static struct { const void *host; char name[512]; } known[4096];
static int n_known, n_launched;
static struct { const char *name; unsigned blocks; } launched[4096];
static struct { dim3 grid, block; size_t lds; void *stream; } pushed;
void __hipRegisterFunction(void **module, const void *host, char *function, const char *name, unsigned limit, void *a, void *b, void *c, void *d, int *e)
{
    (void)module; (void)function; (void)limit; (void)a; (void)b; (void)c; (void)d; (void)e;
    known[n_known].host = host;
    strncpy(known[n_known++].name, name, 511);
}
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipGetLastError(void) { return 0; }
int hipFuncSetAttribute(const void *kernel, int attribute, int value) { (void)kernel; (void)attribute; return value > 160 * 1024; }
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, void *stream)
{
    pushed.grid = grid; pushed.block = block; pushed.lds = lds; pushed.stream = stream;
    return 0;
}
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, void **stream)
{
    *grid = pushed.grid; *block = pushed.block; *lds = pushed.lds; *stream = pushed.stream;
    return 0;
}
int hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t lds, void *stream)
{
    (void)block; (void)args; (void)lds; (void)stream;
    for (int i = 0; i < n_known; ++i)
        if (known[i].host == kernel && n_launched < 4096) { launched[n_launched].name = known[i].name; launched[n_launched++].blocks = grid.x * grid.y * grid.z; }
    return 0;
}
void test_clear(void) { n_launched = 0; }
int test_count(void) { return n_launched; }
const char *test_name(int i) { return launched[i].name; }
unsigned test_blocks(int i) { return launched[i].blocks; }
"""

CALLS = r"""
import ctypes, json, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
runtime.test_name.restype = ctypes.c_char_p
cxx = ctypes.CDLL("libstdc++.so.6")
cxx.__cxa_demangle.restype = ctypes.c_char_p
lib = ctypes.CDLL(sys.argv[2])
i64, vp, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
class Shape(ctypes.Structure):
    _fields_ = [(k, i64) for k in ("N", "K", "C", "ld_phi", "ld_w", "ld_dphi", "ld_dw")] + [("bf16", ctypes.c_int32), ("gradients", ctypes.c_int32)]
lib.rfsf_softmax_xent_workspace_bytes.argtypes = [vp] * 3
lib.rfsf_softmax_xent.argtypes = [vp] * 9 + [sz, vp]
NEVER_READ = 1 << 40
out = []
for N, K, C, bf16, gradients, share in json.loads(sys.argv[3]):
    shape, most, least = Shape(N, K, C, K, K, K, K, bf16, gradients), sz(), sz()
    assert lib.rfsf_softmax_xent_workspace_bytes(ctypes.byref(shape), ctypes.byref(most), ctypes.byref(least)) == 0
    runtime.test_clear()
    p = NEVER_READ
    assert lib.rfsf_softmax_xent(ctypes.byref(shape), p, p, p, None, p, p, p, p, max(least.value, int(share * most.value)), None) == 0
    names = [runtime.test_name(i) for i in range(runtime.test_count())]
    status = ctypes.c_int()
    out.append([cxx.__cxa_demangle(n, None, None, ctypes.byref(status)).decode().replace("(anonymous namespace)::", "").replace("rfsf::", "") for n in names])
print(json.dumps(out))
"""


def of_softmax_xent(tmp_path, calls):
    """Names of the kernels, in order, of calls (N, K, C, bf16, gradients, share of the recommended workspace)."""
    source, runtime = tmp_path / "runtime.c", tmp_path / "libruntime.so"
    source.write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(runtime), str(source)], check=True)
    binding.load_library()
    env = dict(os.environ, HIP_VISIBLE_DEVICES="")
    calls = [[int(v) for v in c[:5]] + [float(c[5] if len(c) > 5 else 1.0)] for c in calls]
    return json.loads(subprocess.run([sys.executable, "-c", CALLS, str(runtime), binding.lib_path(), json.dumps(calls)], env=env, check=True, capture_output=True,
                                     text=True).stdout.strip().splitlines()[-1])
