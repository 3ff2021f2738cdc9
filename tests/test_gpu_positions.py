"""Positions (rope, kv_append_rope into 16-bit and fp32 caches; csrc/rope_append.hip) against the oracle in 64 bits.

Tolerance.  The angle is reduced to r half turns in 64 bits and rounded to fp32, |r| <= 1: off by pi 2^-24 |r| at most (2^-22.3).  The
library's sine and cosine of it are good to 2 units of 2^-24 relative to 1 (2^-23), their product with attn_factor rounds once more
(2^-24), then a product, a sum of products (one rounding each): in all at most (2^-22.3 + 2^-23 + 3 * 2^-24) (|a| + |b|) < 2^-21
(|a| + |b|) attn_factor.  What is stored in 16 bits is rounded once: half a step on top."""
import numpy as np
import pytest

from oracle import positions as P
from tests.ragged_rows import HALF_STEP, LEAST, dev, host, ints, store, table, tree, widen
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

SHAPES = [
    # ctx_lens, spec_lens, tree
    ([1], [0], False),
    ([60000, 1, 17, 16, 33, 5, 2], [0, 0, 16, 15, 1, 4, 1], False),
    ([300, 64, 40, 70], [63, 0, 17, 30], True),
    ([1000, 15, 131072, 1048576], [700, 14, 3, 1], False),
]
HEADS = [(1, 1, 64), (8, 2, 128), (7, 7, 64), (6, 2, 96), (4, 1, 256), (3, 3, 8)]


def frequencies(rot, base=500000.0):
    return (base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)


def close(got, ref, x, rot, dtype, inter, gain):
    """got against ref (turned x), entry by entry"""
    a_at, b_at = P._pairs(rot, inter)
    size = np.zeros_like(ref)
    both = (np.abs(x[..., a_at]) + np.abs(x[..., b_at])) * gain
    size[..., a_at], size[..., b_at] = both, both
    tol = 2.0 ** -21 * size
    tol = tol + HALF_STEP[dtype] * (np.abs(ref) + tol) + LEAST[dtype]
    tol[..., rot:] = 0.0                                    # those stay as they are
    err = np.abs(got - ref)
    assert (err <= tol).all(), (err.max(), (err / np.maximum(tol, 1e-300)).max())


def rots(d):
    return sorted({d, max(2, d // 2), 2, max(2, d - 6), min(d, 20)})


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{len(s[0])}-k{max(s[1])}")
def test_rope(shape, heads, dtype, pkg):  # noqa: F811
    import torch
    ctx, spec, is_tree = shape
    H, _, d = heads
    rng = np.random.default_rng(sum(ctx) + d)
    TQ = sum(spec) + len(spec)
    x = store(rng.normal(0, 2, (TQ, H, d)), dtype)
    parents = tree(rng, spec) if is_tree else None
    for inter in (False, True):
        for n, rot in enumerate(rots(d)):
            f, gain = frequencies(rot), (1.0, 1.25)[n % 2]
            print(f"[case] rope {dtype} {H}x{d} rot={rot} inter={inter} B={len(ctx)}", flush=True)
            kw = dict(max_spec_len=max(spec) + n % 3, interleaved=inter, attn_factor=gain)
            if is_tree:
                kw |= dict(parents=dev(parents), max_spec_len=min(63, max(spec) + n))
            xd, fd = dev(x, dtype), dev(f)
            y = pkg.rope(xd, fd, ints(*ctx), ints(*spec), **kw)
            ref = P.rope(x, f, ctx, spec, dtype=dtype, interleaved=inter, attn_factor=gain, parents=parents)
            close(widen(host(y, dtype), dtype), ref, widen(x, dtype), rot, dtype, inter, gain)
            # in place, and between slices of wider rows: the same bits, and nothing beside them
            wide = torch.full((TQ, (H + 3) * d), 7.0, dtype=xd.dtype, device="cuda")
            part = wide[:, d:(H + 1) * d].unflatten(1, (H, d))
            assert pkg.rope(xd, fd, ints(*ctx), ints(*spec), out=part, **kw) is part
            assert torch.equal(part, y) and bool((wide[:, :d] == 7).all()) and bool((wide[:, (H + 1) * d:] == 7).all())
            part.copy_(xd)
            assert torch.equal(pkg.rope(part, fd, ints(*ctx), ints(*spec), out=part, **kw), y) and bool((wide[:, :d] == 7).all())
            torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("shape", SHAPES[:3], ids=lambda s: f"B{len(s[0])}-k{max(s[1])}")
def test_append(shape, heads, dtype, pkg):  # noqa: F811
    import torch
    ctx, spec, is_tree = shape
    ctx = [min(L, 3000) for L in ctx]
    hq, hkv, d = heads
    rng = np.random.default_rng(sum(ctx) + d)
    TQ = sum(spec) + len(spec)
    bt, num = table(rng, ctx)
    qkv = store(rng.normal(0, 2, (TQ, (hq + 2 * hkv) * d)), dtype)
    q, k, v = (x.reshape(TQ, -1, d) for x in np.split(qkv, [hq * d, (hq + hkv) * d], axis=1))
    pages = [store(rng.normal(0, 1, (num, hkv, 16, d)), dtype) for _ in range(2)]
    parents = tree(rng, spec) if is_tree else None
    where = [(bt[i, t // 16], t % 16) for _, i, t in P.row_positions(ctx, spec)]
    for inter in (False, True):
        for n, rot in enumerate(rots(d)):
            f, gain = frequencies(rot), (1.0, 0.75)[n % 2]
            print(f"[case] append {dtype} {heads} rot={rot} inter={inter} B={len(ctx)}", flush=True)
            kw = dict(max_spec_len=max(spec), interleaved=inter, attn_factor=gain, parents=dev(parents) if is_tree else None)
            kp, vp, wide = dev(pages[0], dtype), dev(pages[1], dtype), dev(qkv, dtype)
            qd, kd, vd = (x.unflatten(1, (-1, d)) for x in wide.split([hq * d, hkv * d, hkv * d], dim=1))
            args = (dev(f), kp, vp, dev(bt), ints(*ctx), ints(*spec))
            out = pkg.kv_append_rope(qd, kd, vd, *args, **kw)
            assert out.is_contiguous() and torch.equal(out, pkg.rope(qd, args[0], *args[4:], **kw))
            turned = widen(host(pkg.rope(kd, args[0], *args[4:], **kw), dtype), dtype)
            ref = P.rope(k, f, ctx, spec, dtype=dtype, interleaved=inter, attn_factor=gain, parents=parents)
            close(turned, ref, widen(k, dtype), rot, dtype, inter, gain)
            # the cache: the turned keys and the values, bit for bit, and nothing else
            want_k, want_v = widen(pages[0], dtype), pages[1].copy()
            for row, (p, slot) in enumerate(where):
                want_k[p, :, slot], want_v[p, :, slot] = turned[row], v[row]
            assert np.array_equal(widen(host(kp, dtype), dtype), want_k) and np.array_equal(host(vp, dtype), want_v)
            # queries in place (beside the keys and values), and none at all
            kp2, vp2 = dev(pages[0], dtype), dev(pages[1], dtype)
            assert pkg.kv_append_rope(None, kd, vd, args[0], kp2, vp2, *args[3:], **kw) is None
            assert torch.equal(kp2, kp) and torch.equal(vp2, vp)
            assert torch.equal(pkg.kv_append_rope(qd, kd, vd, *args, q_out=qd, **kw), out) and torch.equal(kp2, kp)
    # nothing turned: kv_append
    kp, vp, kp2, vp2 = (dev(pages[i % 2], dtype) for i in range(4))
    kc, vc = dev(k, dtype), dev(v, dtype)
    pkg.kv_append(kc, vc, kp, vp, dev(bt), ints(*ctx), ints(*spec), max_spec_len=max(spec))
    pkg.kv_append_rope(None, kc, vc, None, kp2, vp2, dev(bt), ints(*ctx), ints(*spec), max_spec_len=max(spec))
    assert torch.equal(kp, kp2) and torch.equal(vp, vp2)


@pytest.mark.parametrize("bits", [16, 8])
def test_the_most_query_heads_per_kv_head(bits, pkg):  # noqa: F811
    """As many units per workgroup as there may be: 255 query heads of 256 channels, two kv heads, one pair turned."""
    import torch
    ctx, spec, hkv, d = [40, 16], [31, 15], 2, 256
    q = torch.randn((48, 255 * hkv, d), device="cuda").half()
    k, v = (torch.randn((48, hkv, d), device="cuda").half() for _ in range(2))
    kind = torch.float8_e4m3fn if bits == 8 else torch.half
    pools = [torch.zeros((4, hkv, 16, d), device="cuda").to(kind) for _ in range(2)]
    scales = [torch.ones((4, hkv), device="cuda") for _ in range(2)] if bits == 8 else [None] * 2
    f, bt = frequencies(2), dev(np.array([[2, 0, 1], [3, -1, -1]], np.int32))
    out = pkg.kv_append_rope(q, k, v, dev(f), *pools, bt, ints(*ctx), ints(*spec), max_spec_len=31, k_scales=scales[0], v_scales=scales[1])
    close(widen(host(out), "f16"), P.rope(host(q), f, ctx, spec, dtype="f16"), widen(host(q), "f16"), 2, "f16", False, 1.0)
    if bits == 16:
        assert torch.equal(pools[1][3].transpose(0, 1), v[32:])


def test_far_positions_and_fast_pairs(pkg):  # noqa: F811
    """Angles of 10^9 radians: what 32 bits would make of them is noise."""
    L = (1 << 30) - 1
    x = store(np.random.default_rng(3).normal(size=(3, 2, 64)), "f32")
    f = np.linspace(0.9, 1.1, 32).astype(np.float32)
    y = pkg.rope(dev(x), dev(f), ints(L), ints(2), max_spec_len=2)
    close(host(y).astype(np.float64), P.rope(x, f, [L], [2], dtype="f32"), x.astype(np.float64), 64, "f32", False, 1.0)


def test_not_finite_entries_stay_in_their_pairs(pkg):  # noqa: F811
    x = np.ones((2, 3, 64), np.float32)
    x[0, 1, 5], x[1, 2, 40], x[1, 0, 63] = np.nan, np.inf, -np.inf
    y = host(pkg.rope(dev(x), dev(frequencies(32)), ints(9), ints(1), max_spec_len=1))
    bad = np.zeros(x.shape, bool)
    bad[0, 1, [5, 21]] = True
    assert np.array_equal(~np.isfinite(y[..., :32]), bad[..., :32]) and np.array_equal(y[..., 32:], x[..., 32:])


def test_lengths_that_make_no_sense_are_left_alone(pkg):  # noqa: F811
    """A context shorter than its rows, and a table whose entries are outside the pool or behind its width."""
    import torch
    f = dev(frequencies(64))
    q, k, v = (torch.randn((8, h, 64), device="cuda").bfloat16() for h in (4, 2, 2))
    kp, vp = (torch.zeros((6, 2, 16, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    out = torch.full_like(q, 7.0)
    bt = dev(np.array([[0, 9], [-5, 6], [2, 1]], np.int32))
    # request 0: fewer tokens than rows; 1: both pages outside the pool; 2: fine up to the end of its table
    pkg.kv_append_rope(q, k, v, f, kp, vp, bt, ints(1, 17, 34), ints(2, 1, 2), max_spec_len=2, q_out=out)
    torch.cuda.synchronize()
    assert bool((out[:3] == 7).all()) and not bool((out[3:] == 7).any())
    assert bool((kp[[0, 1, 3, 4, 5]][:, :, :15] == 0).all()) and bool((kp[2] == 0).all())
    assert torch.equal(vp[1, :, 15], v[5]) and bool((vp[1, :, :15] == 0).all())
    # more rows claimed than there are
    out.fill_(7.0)
    pkg.rope(q, f, ints(30, 30, 30), ints(2, 2, 2), max_spec_len=2, out=out)
    assert bool((out[6:] == 7).all()) and not bool((out[:6] == 7).any())


@pytest.mark.parametrize("bits", [16, 8])
def test_lengths_at_the_ends_of_32_bits(bits, pkg):  # noqa: F811
    """Several chunks of rows behind a position whose next ones do not fit in 32 bits: turned, and no page is written to."""
    import torch
    d, most, low = 64, 2 ** 31 - 1, -2 ** 31
    f = frequencies(d, 10.0) / np.float32(64)           # (2^31 steps of 1 are more turns than 64 bits hold to 2^-21)
    ctx, spec = [most, low, most - 20, 40, low + 30, most], [40, 40, 5, 40, 60, 0]
    TQ = sum(spec) + len(spec)
    q, k, v = (torch.randn((TQ, 2, d), device="cuda").half() for _ in range(3))
    kind = torch.float8_e4m3fn if bits == 8 else torch.half
    pools = [torch.zeros((4, 2, 16, d), device="cuda").to(kind) for _ in range(2)]
    scales = [torch.ones((4, 2), device="cuda") for _ in range(2)] if bits == 8 else [None] * 2
    out, table_ = torch.full_like(q, 7.0), torch.full((6, 3), 2, dtype=torch.int32, device="cuda")
    pkg.kv_append_rope(q, k, v, dev(f), *pools, table_, ints(*ctx), ints(*spec), max_spec_len=62, k_scales=scales[0], v_scales=scales[1], q_out=out)
    torch.cuda.synchronize()
    assert all(bool((x.float() == 0).all()) for x in pools) and all(bool((x == 1).all()) for x in scales if x is not None)
    row = 0
    for L, s in zip(ctx, spec):
        part = slice(row, row + s + 1)
        if L < s + 1:                                       # no such request
            assert bool((out[part] == 7).all())
        else:
            close(widen(host(out[part]), "f16"), P.rope(host(q[part]), f, [L], [s], dtype="f16"), widen(host(q[part]), "f16"), d, "f16", False, 1.0)
        row += s + 1
    assert torch.equal(pkg.rope(q, dev(f), ints(*ctx), ints(*spec), max_spec_len=62, out=torch.full_like(q, 7.0)), out)


def test_many_requests_on_streams_and_in_graphs(pkg):  # noqa: F811
    import torch
    rng = np.random.default_rng(8)
    ctx = [int(x) for x in rng.integers(9, 200, 700)]
    spec = [int(x) for x in rng.integers(0, 9, 700)]
    bt, num = table(rng, ctx)
    TQ = sum(spec) + 700
    q, k, v = (torch.randn((TQ, h, 64), device="cuda").half() for h in (6, 2, 2))
    f = dev(frequencies(64))
    kp, vp = (torch.zeros((num, 2, 16, 64), device="cuda", dtype=torch.half) for _ in range(2))
    args = (f, kp, vp, dev(bt), ints(*ctx), ints(*spec))
    out = pkg.kv_append_rope(q, k, v, *args, max_spec_len=8)
    ref = P.rope(host(q), host(f), ctx, spec, dtype="f16")
    close(widen(host(out), "f16"), ref, widen(host(q), "f16"), 64, "f16", False, 1.0)
    want, want_k = out.clone(), kp.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    kp.zero_()
    torch.cuda.synchronize()
    other = pkg.kv_append_rope(q, k, v, *args, max_spec_len=8, stream=stream)
    stream.synchronize()
    assert torch.equal(other, want) and torch.equal(kp, want_k)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = pkg.kv_append_rope(q, k, v, *args, max_spec_len=8)
    for n in range(3):
        kp.zero_()
        held.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want) and torch.equal(kp, want_k)
        assert torch.equal(pkg.rope(q, f, args[4], args[5], max_spec_len=8), want)
