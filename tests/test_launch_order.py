"""What a call enqueues, and in which order, without a GPU: functions of this file in the place of the HIP runtime, in a process of
their own."""
import os
import subprocess
import sys

import pytest

from paper_2503_05096_amd import binding
from paper_2503_05096_amd.build import LIB_PATH

RUNTIME = r"""
#include <stdio.h>
#include <stddef.h>
#include <stdlib.h>
static struct { const void *host; char *name; } known[65536];
static int n_known;
typedef struct { unsigned x, y, z; } dim3_t;
void *handle;
void **__hipRegisterFatBinary(const void *data) { return &handle; }
void __hipUnregisterFatBinary(void **m) {}
void __hipRegisterVar() {}
void __hipRegisterFunction(void **m, const void *host, char *device, const char *name) { known[n_known].host = host; known[n_known++].name = device; }
int __hipPushCallConfiguration(dim3_t g, dim3_t b, size_t shared, void *stream) { return 0; }
int __hipPopCallConfiguration(dim3_t *g, dim3_t *b, size_t *shared, void **stream) { return 0; }
int hipLaunchKernel(const void *f, dim3_t g, dim3_t b, void **args, size_t shared, void *stream)
{
    for (int i = 0; i < n_known; ++i) if (known[i].host == f) { printf("%s\n", known[i].name); return 0; }
    printf("unknown kernel\n");
    return 0;
}
int hipEventRecord(void *e, void *stream) { printf("event %p on %p\n", e, stream); return 0; }
int hipGetLastError(void) { return 0; }
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int *v, int attr, int dev) { *v = 256; return 0; }
int hipFuncSetAttribute(const void *f, int attr, int v) { return 0; }
int hipGetSymbolAddress(void **p, const void *symbol) { *p = (void *)0x1000; return 0; }
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *f, int block, size_t shared) { *n = 2; return 0; }
"""

CALL = """
import ctypes as C, sys
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
L = C.CDLL(sys.argv[2])
class Dims(C.Structure):
    _fields_ = [(n, C.c_float if n == "scale" else C.c_void_p if n.startswith("timing") else C.c_int32) for n in sys.argv[3].split(",")]
d = Dims()
for item in sys.argv[4].split(","):
    name, value = item.split("=")
    setattr(d, name, int(value))
p = [C.c_void_p(0x100000000 * (k + 1)) for k in range(11)]
if sys.argv[5] == "remap":
    rc = L.adaspec_kv_remap(*p[:10], C.byref(d), p[10], C.c_size_t(1 << 40), C.c_void_p(0x77))
elif sys.argv[5] == "window":
    rc = L.adaspec_verify_attn_window(*p[:7], C.byref(d), C.c_int32(3000), C.c_int32(4), p[7], C.c_size_t(1 << 30), C.c_void_p(0x77))
else:
    rc = L.adaspec_verify_attn(*p[:7], C.byref(d), p[7], C.c_size_t(1 << 30), C.c_void_p(0x77))
sys.exit(-rc)
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    at = tmp_path_factory.mktemp("runtime")
    (at / "hip.c").write_text(RUNTIME)
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-w", "-o", str(at / "libhip_stub.so"), str(at / "hip.c")], check=True)
    return str(at / "libhip_stub.so")


def lines(runtime, which, fields, dims):
    """what the library's call of these dims enqueues"""
    r = subprocess.run([sys.executable, "-c", CALL, runtime, LIB_PATH, ",".join(n for n, _ in fields), ",".join(f"{k}={v}" for k, v in dims.items()),
                        which], capture_output=True, text=True, timeout=120, env={**os.environ, "PYTHONPATH": ""})
    assert r.returncode == 0, r.stderr
    return [line for line in r.stdout.split("\n") if line]


def enqueued(runtime, which, **kw):
    base = dict(batch=1, total_q=6, max_spec_len=5, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, num_pages=4096, max_pages_per_req=4000,
                dtype=binding.BF16, out_dtype=binding.BF16, timing_start=0xa0, timing_stop=0xb0)
    base.update(kw)
    return [line if line.startswith("event") else "combine" if "combine" in line else "plan" if "plan" in line else "main" if "attn" in line else line
            for line in lines(runtime, which, binding.AttnDims._fields_, base)]


START, STOP = "event 0xa0 on 0x77", "event 0xb0 on 0x77"


@pytest.mark.parametrize("kw", [dict(), dict(head_dim=64), dict(dtype=binding.F32, out_dtype=binding.F32)], ids=str)
def test_events_of_a_windowed_call_in_parts(runtime, kw):
    """As the header says: around the main kernel, without the joining of its parts."""
    assert enqueued(runtime, "window", **kw) == [START, "main", STOP, "combine"]
    assert enqueued(runtime, "window", timing_stop=0, **kw) == ["main", "combine"]


def test_events_of_other_windowed_calls(runtime):
    for kw in (dict(batch=300, total_q=900), dict(path=1), dict(batch=300, total_q=900, path=1)):
        assert enqueued(runtime, "window", **kw) == [START, "main", STOP]


def test_events_of_calls_without_a_window(runtime):
    got = enqueued(runtime, "plain", batch=4, total_q=24)
    assert got.index(START) + 1 == got.index("main") == got.index(STOP) - 1 and set(got[:got.index(START)]) <= {"plan"}
    assert set(got[got.index(STOP) + 1:]) <= {"combine"}


@pytest.mark.parametrize("pages,rows,width,small", [
    (65536, 64, 768, True), (65536, 64, 769, False), (65536, 1024, 48, True), (65536, 1025, 4, False),
    (1 << 19, 64, 768, True), (1 << 19, 1024, 36, True), (1 << 19, 1024, 40, False),
    (1 << 20, 64, 400, True), (1 << 20, 64, 500, False), (1 << 21, 64, 180, True), (1 << 21, 64, 256, False), (1 << 21, 16, 3000, False),
    (1 << 24, 64, 16, True), (1 << 24, 64, 32, False), (1 << 24, 1, 2000, False),
])
def test_form_of_remap(runtime, pages, rows, width, small):
    """Two launches, of which every workgroup of the first reads the whole old table: only where that is not read too often."""
    dims = dict(batch=rows, old_batch=rows, max_pages_per_req=width, num_pages=pages, page_size=16, window=0, sinks=0)
    got = [next(n for n in ("small", "start", "rows", "count", "assign") if n in line) for line in lines(runtime, "remap", binding.PagesDims._fields_, dims)]
    assert got == (["small", "assign"] if small else ["start", "rows", "count", "assign"])
