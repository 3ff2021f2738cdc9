"""What attention over a cache in 8 bits enqueues, without a GPU (the stand-in of test_launch_order): small batches of requests are cut into equal
parts without a metadata kernel, but not where one long request could keep everybody waiting for its few units."""
import os
import subprocess
import sys

import pytest

from paper_2503_05096_amd import binding
from paper_2503_05096_amd.build import LIB_PATH
from tests.test_launch_order import runtime  # noqa: F401  (fixture)

CALL = """
import ctypes as C, sys
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
L = C.CDLL(sys.argv[2])
class Dims(C.Structure):
    _fields_ = [(n, C.c_float if n == "scale" else C.c_void_p if n.startswith("timing") else C.c_int32) for n in sys.argv[3].split(",")]
for case in sys.argv[4].split(";"):
    d = Dims()
    for item in case.split(","):
        name, value = item.split("=")
        setattr(d, name, int(value))
    p = [C.c_void_p(0x100000000 * (k + 1)) for k in range(11)]
    rc = L.adaspec_verify_attn_scaled(*p[:8], None, p[8], C.byref(d), p[9], C.c_size_t(1 << 40), C.c_void_p(0x77))
    assert rc == 0, rc
    C.CDLL(None).puts(b"end")
"""


def enqueued(runtime, cases):  # noqa: F811
    text = []
    for B, tokens, hq, hkv, d in cases:
        dims = dict(batch=B, total_q=7 * B, max_spec_len=6, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=16, num_pages=1 << 20,
                    max_pages_per_req=tokens // 16, dtype=binding.BF16, out_dtype=binding.BF16)
        text.append(",".join(f"{k}={v}" for k, v in dims.items()))
    r = subprocess.run([sys.executable, "-c", CALL, runtime, LIB_PATH, ",".join(n for n, _ in binding.AttnDims._fields_), ";".join(text)],
                       capture_output=True, text=True, timeout=120, env={**os.environ, "PYTHONPATH": ""})
    assert r.returncode == 0, r.stderr
    calls = r.stdout.split("end\n")[:-1]
    assert len(calls) == len(cases)
    return ["plan" in c.split("\n")[0] for c in calls]


@pytest.mark.parametrize("case,metadata", [
    # requests, tokens under the block table, heads, kv heads, head_dim
    ((1, 131072, 32, 8, 128), False), ((2, 131072, 32, 8, 128), False),
    ((4, 65536, 32, 8, 128), False), ((4, 131072, 32, 8, 128), True),
    ((8, 16384, 32, 8, 128), False), ((8, 32768, 32, 8, 128), True), ((8, 65536, 32, 8, 128), True),
    ((16, 8192, 32, 8, 128), False), ((16, 16384, 32, 8, 128), True), ((16, 65536, 32, 8, 128), True),
    ((8, 65536, 16, 2, 128), False), ((32, 65536, 16, 2, 128), True),
    ((8, 20000, 32, 8, 64), False), ((8, 65536, 32, 8, 64), True),
    ((32, 8192, 32, 8, 128), True),
], ids=str)
def test_equal_parts_only_where_those_of_the_longest_request_are_short(runtime, case, metadata):  # noqa: F811
    assert enqueued(runtime, [case]) == [metadata]
