"""Which kernels the host sends calls of include/topoep_ffn.h to, and with what
grids, without a GPU: a process of its own loads a stand-in for the HIP runtime
in front of it, which notes every launch and makes none."""
import json
import os
import re
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_35481_amd", "libtopoep.so")
F32, BF16, F16 = 0, 1, 2

RUNTIME = r"""
#include <stddef.h>
#include <stdint.h>
#include <string.h>
typedef struct { uint32_t x, y, z; } dim3;
enum { KERNELS = 8192, LAUNCHES = 64 };
static const void *address[KERNELS];
static const char *name[KERNELS];
static int kernels, launches;
static struct { const char *name; dim3 grid, block; } seen[LAUNCHES];
static dim3 grid_now, block_now;
void **__hipRegisterFatBinary(const void *data) { static void *handle; (void)data; return &handle; }
void __hipUnregisterFatBinary(void **modules) { (void)modules; }
void __hipRegisterVar(void **m, void *v, char *h, char *d, int e, size_t s, int c, int g) {
  (void)m, (void)v, (void)h, (void)d, (void)e, (void)s, (void)c, (void)g;
}
void __hipRegisterFunction(void **m, const void *host, char *d, const char *device, unsigned t, void *a, void *b,
                           dim3 *c, dim3 *e, int *w) {
  (void)m, (void)d, (void)t, (void)a, (void)b, (void)c, (void)e, (void)w;
  if (kernels < KERNELS) address[kernels] = host, name[kernels++] = strdup(device);
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, void *stream) {
  (void)lds, (void)stream;
  grid_now = grid, block_now = block;
  return 0;
}
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, void **stream) {
  *grid = grid_now, *block = block_now, *lds = 0, *stream = 0;
  return 0;
}
int hipLaunchKernel(const void *host, dim3 grid, dim3 block, void **args, size_t lds, void *stream) {
  (void)args, (void)lds, (void)stream;
  for (int i = 0; i < kernels; ++i)
    if (address[i] == host && launches < LAUNCHES) {
      seen[launches].name = name[i], seen[launches].grid = grid, seen[launches].block = block;
      ++launches;
      return 0;
    }
  return 1;
}
int hipGetLastError(void) { return 0; }
int hipFuncSetAttribute(const void *f, int a, int v) { (void)f, (void)a, (void)v; return 0; }
int taken(void) { const int n = launches; launches = 0; return n; }
const char *taken_name(int i) { return seen[i].name; }
void taken_shape(int i, uint32_t *to) { memcpy(to, &seen[i].grid, 12), memcpy(to + 3, &seen[i].block, 12); }
int all(void) { return kernels; }
const char *all_name(int i) { return name[i]; }
"""

CHILD = r"""
import ctypes, json, sys
runtime = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
runtime.taken_name.restype = runtime.all_name.restype = ctypes.c_char_p
P, I32, I64, SIZE = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
at = lambda n: P(n << 20)                      # (placeholders: aligned, never read)
words = lambda *v: (ctypes.c_int32 * len(v))(*v)

class Rows(ctypes.Structure):
    _fields_ = [(n, P) for n in ("offsets", "pairs", "places", "weights")] + [("k", I32), ("E", I32)]

def call(c):
    op, most = c["op"], SIZE(1 << 62)
    if op in ("forward", "backward"):
        f = words(c["H"], c["I"], c["L"], c["dtype"])
        rows = ctypes.byref(Rows(1 << 20, 2 << 20, 3 << 20, 4 << 20, c["k"], c["E"])) if c["k"] else None
        if op == "forward":
            return lib.topoep_ffn_forward(f, at(5), I64(c["H"]), I32(c["T"]), rows, at(6), at(7), at(8),
                                          at(9) if c["save"] else None, at(10), most, None)
        want = [at(11 + i) if n in c["want"] else None for i, n in enumerate(("x", "weights", "up", "down"))]
        return lib.topoep_ffn_backward(f, at(5), I64(c["H"]), I32(c["T"]), rows, at(6), at(7), at(9), at(8), *want,
                                       at(10), most, None)
    if op == "int8":
        p = words(c["N"], c["K"], max(1, c["groups"]), int(c["gated"]), c["dtype"])
        return lib.topoep_matmul_int8(p, at(1), I64(c["K"]), at(2), I32(c["M"]), at(3) if c["groups"] else None,
                                      I32(0), at(4), at(5), at(6), at(7), most, None)
    if op == "quantize":
        return lib.topoep_quantize(at(1), I32(c["dtype"]), I64(c["ld"]), I32(c["M"]), I32(c["K"]), at(2), at(3), None)
    return lib.topoep_expert_rows(at(1), I32(c["T"]), I32(c["k"]), None, I32(c["L"]), I32(c["L"]), at(2), at(3), at(4),
                                  at(5), most, None)

answers = []
for c in json.load(sys.stdin):
    rc, shape, got = call(c), (ctypes.c_uint32 * 6)(), []
    for i in range(runtime.taken()):
        runtime.taken_shape(i, shape)
        got.append([runtime.taken_name(i).decode(), list(shape[:3]), list(shape[3:])])
    answers.append([rc, got])
json.dump([answers, [runtime.all_name(i).decode() for i in range(runtime.all())]], sys.stdout)
"""


def plain(names):
    """Kernels' names as the sources have them, without namespaces, arguments and result."""
    out = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True).stdout
    return [re.sub(r"\(anonymous namespace\)::|topoep_dev::|^void ", "", n).split("(")[0] for n in out.splitlines()]


def record(calls, tmp):
    """For every call (return code, [(kernel, grid, block)]), and all kernels of the library."""
    source, runtime = os.path.join(str(tmp), "runtime.c"), os.path.join(str(tmp), "runtime.so")
    with open(source, "w") as f:
        f.write(RUNTIME)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", runtime, source], check=True)
    got = subprocess.run([sys.executable, "-c", CHILD, runtime, LIB], input=json.dumps(calls), capture_output=True,
                         text=True, check=True)
    answers, kernels = json.loads(got.stdout)
    names = dict(zip(kernels, plain(kernels)))
    return ([(rc, [(names[n], tuple(grid), tuple(block)) for n, grid, block in got]) for rc, got in answers],
            sorted(names.values()))


def forward(T, H, I, dtype, L=1, k=0, E=1, save=False):
    return dict(op="forward", T=T, H=H, I=I, L=L, k=k, E=E, dtype=dtype, save=save)


def backward(T, H, I, dtype, L=1, k=0, E=1, want=("x", "weights", "up", "down")):
    return dict(op="backward", T=T, H=H, I=I, L=L, k=k, E=E, dtype=dtype, want=list(want))


def int8(M, N, K, dtype, groups=0, gated=False):
    return dict(op="int8", M=M, N=N, K=K, groups=groups, gated=gated, dtype=dtype)


def quantize(M, K, dtype, ld=None):
    return dict(op="quantize", M=M, K=K, dtype=dtype, ld=ld or K)


def rows(T, k, L):
    return dict(op="rows", T=T, k=k, L=L)
