"""What kv_append_rope leaves in the cache where a workgroup has as many units as there may be: 255 query heads of 256 channels per kv head,
one pair turned, full pages (csrc/rope_append.hip).  Scales and values are the oracle's, bit for bit; so are keys, except that the
byte of a turned one (an fp32 value within 2^-21 (|a| + |b|) of the oracle's) may be its neighbour near the border between the two."""
import numpy as np
import pytest

from oracle import positions as P
from tests.ragged_rows import cache8, dev, host, ints, store, widen
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)
from tests.test_gpu_positions import frequencies

pytestmark = pytest.mark.gpu

CTX, SPEC, HKV, D, PAGES = [40, 16, 5], [31, 15, 0], 2, 256, 5
TABLE = np.array([[2, 0, 1], [3, -1, -1], [4, -1, -1]], np.int32)


def inputs(dtype):
    rng = np.random.default_rng(1)
    TQ = sum(SPEC) + len(SPEC)
    return [store(rng.normal(0, 1, (TQ, h, D)), dtype) for h in (255 * HKV, HKV, HKV)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_wide_cache(inter, dtype, pkg):  # noqa: F811
    import torch
    q, k, v = inputs(dtype)
    f = frequencies(2)
    pools = [dev(store(np.full((PAGES, HKV, 16, D), 3.0), dtype)) for _ in range(2)]
    where = ints(*CTX), ints(*SPEC)
    kw = dict(max_spec_len=31, interleaved=inter)
    out = pkg.kv_append_rope(dev(q), dev(k), dev(v), dev(f), *pools, dev(TABLE), *where, **kw)
    assert torch.equal(out, pkg.rope(dev(q), dev(f), *where, **kw))
    turned = host(pkg.rope(dev(k), dev(f), *where, **kw))
    want_k, want_v = (np.full((PAGES, HKV, 16, D), 3.0, k.dtype) for _ in range(2))
    for row, (_, i, t) in enumerate(P.row_positions(CTX, SPEC)):
        want_k[TABLE[i, t // 16], :, t % 16], want_v[TABLE[i, t // 16], :, t % 16] = turned[row], v[row]
    assert np.array_equal(host(pools[0]), want_k) and np.array_equal(host(pools[1]), want_v)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
def test_cache_of_8_bits(inter, dtype, pkg):  # noqa: F811
    q, k, v = inputs(dtype)
    f, rng = frequencies(2), np.random.default_rng(2)
    (k8, ks), (v8, vs) = cache8(rng, PAGES, HKV, D, 0.3), cache8(rng, PAGES, HKV, D, 0.3)
    pools, scales = [dev(k8, "e4m3"), dev(v8, "e4m3")], [dev(ks), dev(vs)]
    pkg.kv_append_rope(dev(q), dev(k), dev(v), dev(f), *pools, dev(TABLE), ints(*CTX), ints(*SPEC), max_spec_len=31, interleaved=inter,
                       k_scales=scales[0], v_scales=scales[1])
    wk, wv, wks, wvs = P.append_scaled(k, v, f, k8, v8, ks, vs, TABLE, CTX, SPEC, dtype=dtype, interleaved=inter)
    assert np.array_equal(host(scales[0]), wks.astype(np.float32)) and np.array_equal(host(scales[1]), wvs.astype(np.float32))
    assert np.array_equal(host(pools[1], "e4m3"), wv)
    got = host(pools[0], "e4m3")
    turned, (a_at, b_at) = P.rope(k, f, CTX, SPEC, dtype=dtype, interleaved=inter), P._pairs(2, inter)
    raw, near = np.abs(widen(k, dtype)), np.zeros(turned.shape)
    near[..., a_at] = near[..., b_at] = 2.0 ** -21 * (raw[..., a_at] + raw[..., b_at])
    differ = got != wk
    for row, (_, i, t) in enumerate(P.row_positions(CTX, SPEC)):
        page, slot = TABLE[i, t // 16], t % 16
        there = differ[page, :, slot].copy()
        differ[page, :, slot] = False
        mid = (P.E4M3[got[page, :, slot]] + P.E4M3[wk[page, :, slot]]) / 2 * wks[page][:, None]
        assert (np.abs(turned[row] - mid) <= near[row])[there].all()
    assert not differ.any()
