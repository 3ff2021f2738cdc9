"""Windowed verification attention with many units (a lone wavefront each where windows are short) and at the limits between its
forms, against the oracle in 64 bits.  Poison and tolerances are those of test_gpu_attn_window.py."""
import numpy as np
import pytest

from tests.test_gpu_attn_window import check, poisoned, run, step, to_device
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

# Hq, Hkv, longest draft: one, two, three row tiles of 16 rows; two row groups, of 64 rows where windows are longer; one row in a unit
HEADS = [(2, 2, 5), (8, 2, 7), (10, 2, 8), (16, 2, 10), (16, 2, 7), (3, 3, 0)]


def many(seed, batch, hq, hkv, most, d, dtype, longest=420):
    rng = np.random.default_rng(seed)
    spec = rng.integers(0, most + 1, batch)
    ctx = np.maximum(rng.integers(1, longest, batch), spec + 1)
    ctx[:4], spec[:4] = [1, 16, 17, longest], 0
    spec[4] = most
    ctx[4] = max(ctx[4], most + 1)
    return step(seed, ctx.tolist(), spec.tolist(), hq, hkv, d, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}-k{h[2]}")
def test_short_windows(heads, d, dtype, pkg):  # noqa: F811
    hq, hkv, most = heads
    for window, sinks in ((1, 0), (16, 4), (33, 20), (200, 1)):
        check(pkg, poisoned(many(1100 + d, 300, hq, hkv, most, d, dtype), window, sinks), window, sinks, paths=("auto",))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_either_side_of_a_unit_count(dtype, d, pkg):  # noqa: F811
    for batch, window in ((256, 100), (257, 100), (1, 2000), (32, 2000), (33, 2000), (129, 700)):
        longest = 2300 if window > 1000 else 420
        check(pkg, poisoned(many(1200 + batch, max(batch, 5), 4, 2, 3, d, dtype, longest), window, 4), window, 4, paths=("auto",))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 64)])
def test_what_a_row_does_not_see_with_many_units(dtype, d, pkg):  # noqa: F811
    """NaN in a token that the first rows of a request see and later ones do not, and in a draft that only the last two rows
see; rows that see neither are off by the rounding that test_gpu_attn_window.py derives."""
    window, sinks, batch = 20, 2, 270
    tol = 2e-6 + (5 * 2.0 ** -18 if dtype == "bf16" else 0.0)
    rng = np.random.default_rng(9)
    st = step(1300, rng.integers(40, 120, batch).tolist(), rng.integers(4, 8, batch).tolist(), 8, 2, d, dtype)
    clean = run(pkg, st, window, sinks, out_dtype=0)
    bad = np.uint16(0x7FC0) if dtype == "bf16" else np.nan
    sees = []
    for i in range(batch):
        L, n = int(st.ctx_lens[i]), int(st.spec_lens[i]) + 1
        hit = (L - n - window + 3, L - 2) if i % 3 else ()
        for t in hit:
            st.v_pages[st.block_table[i, t // 16], :, t % 16, 1::3] = bad
            st.k_pages[st.block_table[i, t // 16], :, t % 16, 5] = bad
        sees += [any(t <= L - n + j and L - n + j - t < window for t in hit) for j in range(n)]
    out = run(pkg, st, window, sinks, out_dtype=0)
    sees = np.array(sees)
    assert sees.any() and not sees.all()
    assert not np.isfinite(out[sees]).all(axis=(1, 2)).any()
    assert np.abs(out[~sees] - clean[~sees]).max() <= tol


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [24, 128, 136, 248])
def test_portable_form_over_several_turns(d, dtype, pkg):  # noqa: F811
    """Lists of pages that end anywhere in a wavefront's turns, of up to three of them; one row in a unit, and eight."""
    for window, sinks in ((700, 40), (1000, 0), (3, 17)):
        st = step(1500 + d, [1, 63, 64, 65, 257, 900, 700, 513], [0, 1, 0, 2, 3, 6, 0, 5], 6, 2, d, dtype)
        check(pkg, poisoned(st, window, sinks), window, sinks, paths=("vector",))
    st = many(1550 + d, 180, 6, 2, 3, d, dtype)                     # 12 rows: units of eight
    check(pkg, poisoned(st, 90, 4), 90, 4, paths=("vector",))


def test_two_calls_at_once_and_rows_behind_the_last_request(pkg):  # noqa: F811
    """Two streams, a workspace each; outputs with rows behind the last request's, which stay as they were."""
    import torch
    steps = [poisoned(many(1400, 300, 8, 2, 4, 128, "bf16"), 60, 3), poisoned(step(1401, [4000, 900], [4, 2], 8, 2, 128, "bf16"), 3000, 3)]
    jobs = []
    for st, window in zip(steps, (60, 3000)):
        d = to_device(st, acceptance=False)
        q = torch.cat([d.q, torch.full_like(d.q[:3], float("nan"))])
        args = (q, d.k_pages, d.v_pages, d.block_table, d.ctx_lens, d.spec_lens)
        kw = dict(max_spec_len=st.max_spec_len + 1, window=window, sinks=3)     # (total_q is at most batch times that and one)
        ref = pkg.verify_attn(*args, torch.full_like(q, 7.0), **kw)
        torch.cuda.synchronize()
        assert (ref[-3:] == 7.0).all() and torch.isfinite(ref).all()
        jobs.append((args, kw, ref, torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    for _ in range(5):
        for args, kw, ref, ws, stream, outs in jobs:
            with torch.cuda.stream(stream):
                outs.append(pkg.verify_attn(*args, torch.full_like(ref, 7.0), workspace=ws, **kw))
    torch.cuda.synchronize()
    for _, _, ref, _, _, outs in jobs:
        assert all(torch.equal(o, ref) for o in outs)


@pytest.mark.parametrize("dtype,hkv", [("bf16", 8), ("f32", 8)])
def test_a_pool_beyond_32_bits(dtype, hkv, pkg):  # noqa: F811
    """Pages whose byte offsets pass 2^32, and whose values' offsets pass 2^31, give what the same pages give at the pool's
beginning: few units, many (lone wavefronts), and the portable form."""
    import torch
    for batch, longest, window in ((3, 1500, 1000), (90, 200, 60)):
        st = poisoned(many(1600 + batch, max(batch, 5), 2 * hkv, hkv, 2, 128, dtype, longest), window, 4)
        d = to_device(st, acceptance=False)
        used = d.k_pages.shape[0]
        NP = 2 ** 32 // (hkv * 16 * 128 * (2 if dtype == "bf16" else 4)) + 2 * used + 100
        k, v = (torch.empty((NP,) + tuple(d.k_pages.shape[1:]), dtype=d.q.dtype, device="cuda") for _ in range(2))
        at = NP - used
        k[at:], v[at:] = d.k_pages, d.v_pages
        far = torch.where(d.block_table >= 0, d.block_table + at, d.block_table)
        for path in ("auto", "vector"):
            kw = dict(max_spec_len=st.max_spec_len, window=window, sinks=4, path=path)
            ref = pkg.verify_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.ctx_lens, d.spec_lens, **kw)
            out = pkg.verify_attn(d.q, k, v, far, d.ctx_lens, d.spec_lens, **kw)
            assert torch.isfinite(ref).all() and torch.equal(out, ref), (batch, path)
        del k, v
        torch.cuda.empty_cache()
