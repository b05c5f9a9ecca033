"""Which kernels calls of layer norm, its backward pass, dropout and scores with adapters launch, and which there are, without a GPU: as launches.py for softmax cross entropies."""
import json
import os
import subprocess
import sys

from paper_2501_07145_amd import binding
from tests.launches import RUNTIME

ALL = r"""
int test_known(void) { return n_known; }
const char *test_known_name(int i) { return known[i].name; }
"""

CALLS = r"""
import ctypes, json, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
runtime.test_name.restype = runtime.test_known_name.restype = ctypes.c_char_p
cxx = ctypes.CDLL("libstdc++.so.6")
cxx.__cxa_demangle.restype = ctypes.c_char_p
lib = ctypes.CDLL(sys.argv[2])
i64, i32, vp, sz, dbl = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double
class Mask(ctypes.Structure):
    _fields_ = [("p", dbl), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("counter", vp), ("first_row", i64)]
class Norm(ctypes.Structure):
    _fields_ = [(k, i64) for k in ("N", "K", "ld_x", "ld_y", "ld_dx")] + [("bf16", i32)]
class Adapters(ctypes.Structure):
    _fields_ = [(k, i64) for k in ("K", "C", "rank", "count")] + [("bf16", i32)]
lib.rfsf_dropout.argtypes = [vp, vp, i32, i64, i64, i64, vp, i64, vp]
lib.rfsf_layer_norm.argtypes = [vp, vp, vp, vp, dbl, vp, vp, vp, vp, vp]
lib.rfsf_layer_norm_backward.argtypes = [vp] * 11 + [sz, vp]
lib.rfsf_adapted_scores_workspace_bytes.argtypes = [vp, i64, vp, vp]
lib.rfsf_adapted_scores.argtypes = [vp, vp, vp, i64, i64, vp, vp, i64, vp, sz, vp]
P = 1 << 40             # never read
def name(n):
    status = ctypes.c_int()
    n = cxx.__cxa_demangle(n, None, None, ctypes.byref(status)).decode().replace("(anonymous namespace)::", "").replace("rfsf::", "").replace("plane::", "")
    return n.replace("unsigned short", "bf16").replace("void ", "", 1).split("(PlaneMode)")[0].split("(")[0] if "PlaneMode" not in n else n.replace("(PlaneMode)", "").replace("void ", "", 1).split(">(")[0] + ">"
out = []
mask = Mask(0.5, 1, 2, None, 0)
for call in json.loads(sys.argv[3]):
    runtime.test_clear()
    op, a = call[0], call[1:]
    if op == "norm":
        N, K, bf16, drop = a
        s = Norm(N, K, K, K, K, bf16)
        rc = lib.rfsf_layer_norm(ctypes.byref(s), P, P, P, 1e-5, ctypes.byref(mask) if drop else None, P, P, P, None)
    elif op == "back":
        N, K, bf16, drop, dX, gains = a
        s = Norm(N, K, K, K, K, bf16)
        rc = lib.rfsf_layer_norm_backward(ctypes.byref(s), P, P, P, P, P, ctypes.byref(mask) if drop else None, P if dX else None, P if gains else None,
                                          P if gains else None, P, 1 << 50, None)
    elif op == "dropout":
        N, K, bf16 = a
        rc = lib.rfsf_dropout(ctypes.byref(mask), P, bf16, N, K, K, P, K, None)
    else:
        N, K, C, rank, count, bf16, share = a
        s, most, least = Adapters(K, C, rank, count, bf16), sz(), sz()
        assert lib.rfsf_adapted_scores_workspace_bytes(ctypes.byref(s), N, ctypes.byref(most), ctypes.byref(least)) == 0
        rc = lib.rfsf_adapted_scores(ctypes.byref(s), P, P, N, K, P, P, C, P, max(least.value, int(share * most.value)), None)
    assert rc == 0, (call, rc)
    out.append([name(runtime.test_name(i)) for i in range(runtime.test_count())])
print(json.dumps([out, sorted({name(runtime.test_known_name(i)) for i in range(runtime.test_known())})]))
"""


def launches(tmp_path, calls):
    """(names of the kernels that each call launches, in order; all kernels of the library). Calls: ("norm", N, K, bf16, drop), ("back", N, K, bf16, drop, dX, gains),
    ("dropout", N, K, bf16), ("scores", N, K, C, rank, count, bf16, share of the recommended workspace)."""
    source, runtime = tmp_path / "runtime.c", tmp_path / "libruntime.so"
    source.write_text(RUNTIME + ALL)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(runtime), str(source)], check=True)
    binding.load_library()
    calls = [[c[0]] + [float(v) if isinstance(v, float) else int(v) for v in c[1:]] for c in calls]
    return json.loads(subprocess.run([sys.executable, "-c", CALLS, str(runtime), binding.lib_path(), json.dumps(calls)], env=dict(os.environ, HIP_VISIBLE_DEVICES=""),
                                     check=True, capture_output=True, text=True).stdout.strip().splitlines()[-1])
