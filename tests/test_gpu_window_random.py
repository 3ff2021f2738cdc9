"""Windowed attention and the pages of the cache on random shapes, against the oracle.  ADASPEC_SOAK_CASES: cases per kind (default 6).

Tolerance of attention on the fp32 accumulator: 2e-5 for the fp32 arithmetic, as in test_gpu_attn_window.py; with bf16 weights in two
pieces 2^-18 of the largest value on top (values are N(0, 1): random shapes reach some above 5)."""
import os

import numpy as np
import pytest

from oracle.window import verify_attn_window
from tests.test_gpu_attn_window import HALF_STEP, poisoned, run, step
from tests.test_gpu_kv_pages import check_compact, check_remap, state
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

CASES = int(os.environ.get("ADASPEC_SOAK_CASES", 6))


def log_uniform(r, lo, hi):
    return int(round(np.exp(r.uniform(np.log(lo), np.log(hi)))))


@pytest.mark.parametrize("seed", range(CASES))
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_window(dtype, seed, pkg):  # noqa: F811
    r = np.random.default_rng((seed, len(dtype), ord(dtype[0])))
    for _ in range(4):
        B, hkv, G = log_uniform(r, 1, 300), int(r.integers(1, 5)), int(r.choice([1, 1, 2, 3, 4, 5, 7, 8, 16]))
        longest = min(log_uniform(r, 20, 3000), max(20, 40000 // B))
        most = min(int(r.integers(0, 14)), max(0, 6_000_000 // (B * G * hkv * longest) - 1))
        spec = r.integers(0, most + 1, B)
        ctx = np.maximum(r.integers(1, longest + 1, B), spec + 1)
        d = int(r.choice([64, 128, 64, 128, 8 * int(r.integers(1, 33))]))
        window, sinks = log_uniform(r, 1, 4000), int(r.choice([0, 0, 1, 4, 17, int(r.integers(0, 200))]))
        bound = int(spec.max() + r.choice([0, 0, 1, 20]))
        print(f"[case] {dtype} seed={seed} B={B} {G * hkv}/{hkv} k<={most} (bound {bound}) L<={longest} d={d} window={window} sinks={sinks}", flush=True)
        st = poisoned(step(int(r.integers(1 << 30)), ctx.tolist(), spec.tolist(), G * hkv, hkv, d, dtype), window, sinks)
        ref = verify_attn_window(st.q, st.k_pages, st.v_pages, st.block_table, st.ctx_lens, st.spec_lens, window=window, sinks=sinks, dtype=dtype)
        v = (st.v_pages.astype(np.uint32) << 16).view(np.float32) if dtype == "bf16" else st.v_pages
        tol = 2e-5 + (2.0 ** -18 * float(np.nanmax(np.abs(v.astype(np.float32)))) if dtype == "bf16" else 0.0)
        assert np.abs(run(pkg, st, window, sinks, out_dtype=0, max_spec_len=bound) - ref).max() <= tol
        assert (np.abs(run(pkg, st, window, sinks, max_spec_len=bound) - ref) <= tol + HALF_STEP[dtype] * np.abs(ref)).all()


@pytest.mark.parametrize("seed", range(CASES))
def test_pages(seed, pkg):  # noqa: F811
    r = np.random.default_rng((seed, 77))
    for _ in range(4):
        old, B, width, P = int(r.integers(1, 1400)), int(r.integers(1, 2300)), int(r.integers(1, 60)), int(r.choice([1, 2, 16, 16, 64]))
        table, refs, held = state(r, old, width, P, int(r.integers(0, 4000)), extra=int(r.integers(0, 5)))
        lens, sources = np.minimum(r.integers(0, width * P + 1, old), held * P), r.integers(-1, old, B)
        more = np.where(sources >= 0, lens[np.maximum(sources, 0)], 0) + r.integers(-2, 3 * P, B)
        kw = dict(page_size=P)
        if r.random() < 0.5:
            kw.update(window=int(r.integers(1, width * P + 1)), sinks=int(r.integers(0, 3 * P)))
        print(f"[case] pages seed={seed} {old}->{B} x{width} pages={len(refs)} {kw}", flush=True)
        check_remap(pkg, table, refs, sources, lens, more, alias=bool(r.random() < 0.5), **kw)
        check_compact(pkg, table, refs, max_moves=int(r.integers(1, len(refs) + 1)), alias=bool(r.random() < 0.5))
