"""What the gated delta rule's calls do when a kernel is refused the LDS that it needs, without a GPU: the library against a runtime of a dozen functions
that notes which kernels are launched and refuses what it is told to."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2604_25422_amd import _build

RUNTIME = r"""
#include <stddef.h>
#include <string.h>
typedef struct { unsigned x, y, z; } dim3_t;
enum { MANY = 8192 };
static const void *hosts[MANY];
static const char *names[MANY];
static int known, launched, refuse_at = -1, asked, error;
static const char *log_[MANY];
static unsigned long long fat;
void **__hipRegisterFatBinary(const void *x) { (void)x; static void *p = &fat; return &p; }
void __hipUnregisterFatBinary(void **x) { (void)x; }
void __hipRegisterFunction(void **m, const void *host, char *device, const char *name, unsigned a, void *b, void *c, void *d, void *e, int *f)
{ (void)m, (void)device, (void)a, (void)b, (void)c, (void)d, (void)e, (void)f; if (known < MANY) hosts[known] = host, names[known++] = name; }
void __hipRegisterVar(void **m, void *v, char *a, char *b, int c, size_t d, int e, int f) { (void)m, (void)v, (void)a, (void)b, (void)c, (void)d, (void)e, (void)f; }
static struct { dim3_t g, b; size_t s; void *st; } call;
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t s, void *st) { call.g = g, call.b = b, call.s = s, call.st = st; return 0; }
int __hipPopCallConfiguration(dim3_t *g, dim3_t *b, size_t *s, void **st) { *g = call.g, *b = call.b, *s = call.s, *st = call.st; return 0; }
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipGetLastError(void) { int e = error; error = 0; return e; }
int hipFuncSetAttribute(const void *f, int a, int v) { (void)f, (void)a, (void)v; return asked++ == refuse_at ? (error = 1) : 0; }
int hipLaunchKernel(const void *f, dim3_t g, dim3_t b, void **args, size_t s, void *st)
{
    (void)g, (void)b, (void)args, (void)s, (void)st;
    const char *name = "?";
    for (int i = 0; i < known; ++i) if (hosts[i] == f) name = names[i];
    if (launched < MANY) log_[launched++] = name;
    return 0;
}
void test_refuse(int at) { refuse_at = at, asked = launched = 0; }
int test_launched(void) { return launched; }
const char *test_name(int i) { return log_[i]; }
"""

PROGRAM = r"""
import ctypes, json, re, sys
rt = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)       # (in front of the library's own runtime, which is never called)
rt.test_name.restype = ctypes.c_char_p
lib = ctypes.CDLL(sys.argv[2])
class Seq(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_longlong)]
vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
lib.dwconv_delta_fwd.argtypes = [Seq] * 5 + [vp, vp, Seq, vp, vp, vp, sz] + [i] * 6 + [f, f, i, vp]
lib.dwconv_delta_bwd.argtypes = [Seq] * 6 + [vp] * 3 + [Seq] * 3 + [vp] * 4 + [sz] + [i] * 6 + [f, f, i, vp]
P, dims = 0x1000, (1, 2, 2, 128, 128, 8192)
s = lambda: Seq(P, 1 << 30)
fwd = lambda: lib.dwconv_delta_fwd(s(), s(), s(), s(), s(), None, None, s(), P, P, P, 1 << 40, *dims, 1.0, 1e-6, 1, None)
bwd = lambda: lib.dwconv_delta_bwd(s(), s(), s(), s(), s(), s(), P, None, None, s(), s(), s(), P, P, P, P, 1 << 40, *dims, 1.0, 1e-6, 1, None)
out = []
for call in (fwd, bwd):
    for at in (0, 1, 1, -1):
        rt.test_refuse(at)
        rc = call()
        out.append([rc, [re.sub(r".*?(delta_[a-z_]+?)_kernel.*", r"\1", rt.test_name(k).decode()) for k in range(rt.test_launched())]])
print(json.dumps(out))
"""


def test_nothing_is_launched_behind_what_was_refused(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    if _build.is_stale():
        _build.build()
    source, runtime, program = tmp_path / "runtime.c", tmp_path / "runtime.so", tmp_path / "program.py"
    source.write_text(RUNTIME), program.write_text(PROGRAM)
    subprocess.run([gcc, "-shared", "-fPIC", "-O1", "-o", str(runtime), str(source)], check=True)
    r = subprocess.run([sys.executable, str(program), str(runtime), os.path.abspath(_build.LIB_PATH)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    got = json.loads(r.stdout.splitlines()[-1])
    # forward: the spans' walk asks first, then (once that has it) the walk itself; backward the within-chunk kernel too
    fwd = ["delta_pairs", "delta_fwd", "delta_starts", "delta_starts", "delta_starts", "delta_fwd"]
    bwd = ["delta_pairs", "delta_bwd_state", "delta_starts", "delta_starts", "delta_starts", "delta_bwd_state", "delta_bwd_chunk"]
    refused, fine = 7, 0
    assert got[:4] == [[refused, fwd[:1]], [refused, fwd[:5]], [fine, fwd], [fine, fwd]]
    assert got[4:] == [[refused, bwd[:1]], [refused, bwd[:5]], [refused, bwd[:6]], [fine, bwd]]
