"""The cache held in 8 bits: appends, copies of pages, compaction of an accepted path (csrc/rope_append.hip, kv_pages.hip, tree.hip)
against the oracle.  Scales are equal, always.  So are bytes, except of turned keys: their fp32 value is within 2^-21 (|a| + |b|)
of the oracle's (tests/test_gpu_positions.py), so a byte may be its neighbour's where the value is that close to the border
between the two."""
import numpy as np
import pytest

from oracle import positions as P
from tests.ragged_rows import cache8, dev, host, ints, store, table, tree, widen
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)
from tests.test_gpu_positions import HEADS, frequencies, rots

pytestmark = pytest.mark.gpu

SHAPES = [
    # ctx_lens, spec_lens, tree
    ([1], [0], False),
    ([2000, 1, 17, 16, 33, 5, 48, 47], [0, 0, 16, 15, 1, 4, 0, 46], False),
    ([300, 64, 40, 70], [63, 0, 17, 30], True),
    ([500, 90], [400, 3], False),
]


def louder(rng, x, spec, dtype):
    """some rows, heads and entries much larger or smaller than the rest"""
    x = widen(x, dtype)
    x *= 2.0 ** rng.integers(-3, 4, (x.shape[0], x.shape[1], 1))
    x[rng.random(x.shape[:2]) < 0.1] *= 2.0 ** -12
    x[rng.random(x.shape) < 0.002] *= 20.0
    x[rng.random(x.shape[:2]) < 0.05] = 0.0
    return store(x, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{len(s[0])}-k{max(s[1])}")
def test_append(shape, heads, dtype, pkg):  # noqa: F811
    import torch
    ctx, spec, is_tree = shape
    hq, hkv, d = heads
    rng = np.random.default_rng(sum(ctx) + d)
    TQ = sum(spec) + len(spec)
    bt, num = table(rng, ctx)
    q, k, v = (louder(rng, store(rng.normal(0, 1, (TQ, h, d)), dtype), spec, dtype) for h in (hq, hkv, hkv))
    (k8, ks), (v8, vs) = cache8(rng, num, hkv, d), cache8(rng, num, hkv, d, 0.3)
    parents = tree(rng, spec) if is_tree else None
    for inter in (False, True):
        for n, rot in enumerate(rots(d)):
            f, gain = frequencies(rot, 100.0), (1.0, 1.25)[n % 2]
            print(f"[case] append8 {dtype} {heads} rot={rot} inter={inter} B={len(ctx)}", flush=True)
            kw = dict(interleaved=inter, attn_factor=gain)
            dk, dv, dks, dvs = dev(k8, "e4m3"), dev(v8, "e4m3"), dev(ks), dev(vs)
            more = dict(max_spec_len=max(spec), k_scales=dks, v_scales=dvs, parents=dev(parents) if is_tree else None, **kw)
            args = (dev(q, dtype), dev(k, dtype), dev(v, dtype), dev(f), dk, dv, dev(bt), ints(*ctx), ints(*spec))
            out = pkg.kv_append_rope(*args, **more)
            torch.cuda.synchronize()
            assert torch.equal(out, pkg.rope(args[0], args[3], args[7], args[8], max_spec_len=max(spec), parents=more["parents"], **kw))
            wk, wv, wks, wvs = P.append_scaled(k, v, f, k8, v8, ks, vs, bt, ctx, spec, dtype=dtype, parents=parents, **kw)
            assert np.array_equal(host(dks), wks.astype(np.float32)) and np.array_equal(host(dvs), wvs.astype(np.float32))
            assert np.array_equal(host(dv, "e4m3"), wv)
            # keys: near a border the neighbouring code is as good
            got = host(dk, "e4m3")
            turned = P.rope(k, f, ctx, spec, dtype=dtype, parents=parents, **kw)
            a_at, b_at = P._pairs(rot, inter)
            raw, near = np.abs(widen(k, dtype)), np.zeros(turned.shape)
            near[..., a_at] = near[..., b_at] = 2.0 ** -21 * gain * (raw[..., a_at] + raw[..., b_at])
            differ = got != wk
            for row, (_, i, t) in enumerate(P.row_positions(ctx, spec)):
                page, slot = bt[i, t // 16], t % 16
                there = differ[page, :, slot].copy()
                differ[page, :, slot] = False
                if there.any():
                    mid = (P.E4M3[got[page, :, slot]] + P.E4M3[wk[page, :, slot]]) / 2 * wks[page][:, None]
                    assert (np.abs(turned[row] - mid) <= near[row])[there].all()
            assert not differ.any()
            # a second time: every scale covers its page now, and nothing moves
            before = [x.clone() for x in (dk, dv, dks, dvs)]
            pkg.kv_append_rope(None, *args[1:], **more)
            for x, y in zip(before, (dk, dv, dks, dvs)):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # nothing turned
    dk, dv, dks, dvs = dev(k8, "e4m3"), dev(v8, "e4m3"), dev(ks), dev(vs)
    pkg.kv_append(dev(k, dtype), dev(v, dtype), dk, dv, dev(bt), ints(*ctx), ints(*spec), max_spec_len=max(spec), k_scales=dks, v_scales=dvs)
    wk, wv, wks, wvs = P.append_scaled(k, v, None, k8, v8, ks, vs, bt, ctx, spec, dtype=dtype)
    assert np.array_equal(host(dk, "e4m3"), wk) and np.array_equal(host(dv, "e4m3"), wv)
    assert np.array_equal(host(dks), wks.astype(np.float32)) and np.array_equal(host(dvs), wvs.astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_scales_at_their_borders(dtype, pkg):  # noqa: F811
    """Entries of 448 times a power of two and just above, zeros, the smallest and the largest numbers, entries that are not finite."""
    import torch
    d = 64
    tiny = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}[dtype]
    big = {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.38e38}[dtype]
    above = {"f32": 448.0 * (1 + 2.0 ** -23), "f16": 448.25, "bf16": 450.0}[dtype]
    rows = []
    for x in (448.0, above, 447.0, 7.0, 3.5 * (1 + 2.0 ** -10), 0.0, tiny, big, -448.0):
        row = np.zeros(d)
        row[3], row[40] = x, x / 3
        rows.append(row)
    for bad in (np.nan, np.inf, -np.inf):
        row = np.linspace(-3, 3, d)
        row[7] = bad
        rows.append(row)
    with np.errstate(over="ignore"):
        k = store(np.array(rows)[:, None, :], dtype)
    v = k[::-1].copy()
    n = len(rows)
    ctx, spec = [1] * n, [0] * n                         # every row alone in its page
    bt = np.arange(n, dtype=np.int32)[:, None]
    k8, ks = np.zeros((n, 1, 16, d), np.uint8), np.ones((n, 1), np.float32)
    for f, rot in ((frequencies(d), d), (None, 0)):
        dk, dv, dks, dvs = dev(k8, "e4m3"), dev(k8, "e4m3"), dev(ks), dev(ks)
        pkg.kv_append_rope(None, dev(k, dtype), dev(v, dtype), None if f is None else dev(f), dk, dv, dev(bt), ints(*ctx), ints(*spec), max_spec_len=0,
                           k_scales=dks, v_scales=dvs)
        torch.cuda.synchronize()
        with np.errstate(invalid="ignore", over="ignore"):
            wk, wv, wks, wvs = P.append_scaled(k, v, f, k8, k8, ks, ks, bt, ctx, spec, dtype=dtype)
        assert np.array_equal(host(dks), wks.astype(np.float32)) and np.array_equal(host(dvs), wvs.astype(np.float32))
        for got, want in ((host(dk, "e4m3"), wk), (host(dv, "e4m3"), wv)):          # (position 0: turned by nothing, exactly)
            assert np.array_equal(P.E4M3[got], P.E4M3[want], equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_the_largest_entry_beside_one_that_is_not_finite(bad, dtype, pkg):  # noqa: F811
    """It counts, wherever the two are: a value's neighbours, a key's entries that are not turned."""
    import torch
    d = 64
    rows = []
    for at in range(24):
        row = np.full(d, 0.5)
        row[16 + at], row[16 + at + (1 if at % 2 else -1)] = bad, 96.0
        rows.append(row)
    with np.errstate(over="ignore"):
        x = store(np.array(rows)[:, None, :], dtype)
    n = len(rows)
    ctx, spec, bt = [1] * n, [0] * n, np.arange(n, dtype=np.int32)[:, None]
    k8, ks = np.zeros((n, 1, 16, d), np.uint8), np.ones((n, 1), np.float32)
    for f, inter in ((None, False), (frequencies(16), False), (frequencies(16), True)):
        dk, dv, dks, dvs = dev(k8, "e4m3"), dev(k8, "e4m3"), dev(ks), dev(ks)
        pkg.kv_append_rope(None, dev(x, dtype), dev(x, dtype), None if f is None else dev(f), dk, dv, dev(bt), ints(*ctx), ints(*spec), max_spec_len=0,
                           k_scales=dks, v_scales=dvs, interleaved=inter)
        torch.cuda.synchronize()
        with np.errstate(invalid="ignore"):
            wk, wv, wks, wvs = P.append_scaled(x, x, f, k8, k8, ks, ks, bt, ctx, spec, dtype=dtype, interleaved=inter)
        assert (wvs == 0.25).all() and np.array_equal(host(dks), wks.astype(np.float32)) and np.array_equal(host(dvs), wvs.astype(np.float32))
        for got, want in ((host(dk, "e4m3"), wk), (host(dv, "e4m3"), wv)):
            assert np.array_equal(P.E4M3[got], P.E4M3[want], equal_nan=True)


@pytest.mark.parametrize("layers", [None, 3])
def test_copies_of_pages(layers, pkg):  # noqa: F811
    import torch
    rng = np.random.default_rng(4)
    num, hkv, d = 50, 3, 72
    lead = () if layers is None else (layers,)
    pages = [rng.integers(0, 256, lead + (num, hkv, 16, d)).astype(np.uint8) for _ in range(2)]
    scales = [rng.random(lead + (num, hkv)).astype(np.float32) for _ in range(2)]
    src, dst = np.array([3, -1, 49, 7, 7, 60], np.int32), np.array([5, 8, 0, -1, 21, 9], np.int32)
    dp, ds = [dev(x, "e4m3") for x in pages], [dev(x) for x in scales]
    pkg.kv_copy_pages(*dp, dev(src), dev(dst), k_scales=ds[0], v_scales=ds[1])
    torch.cuda.synchronize()
    for x, s, dx, dsx in zip(pages, scales, dp, ds):
        for a, b in ((3, 5), (49, 0), (7, 21)):
            x[..., b, :, :, :], s[..., b, :] = x[..., a, :, :, :], s[..., a, :]
        assert np.array_equal(host(dx, "e4m3"), x) and np.array_equal(host(dsx), s)


@pytest.mark.parametrize("seed", range(6))
def test_compaction_of_an_accepted_path(seed, pkg):  # noqa: F811
    import torch
    rng = np.random.default_rng(100 + seed)
    d, hkv = [(128, 2), (64, 3), (256, 1), (96, 2), (8, 1), (128, 8)][seed]
    spec = [0, 5, 63, 20, 7, 40, 63]
    ctx = [1, 6, 64, 190, 300, 47, 79]
    bt, num = table(rng, ctx)
    lens, path = [], np.full((len(spec), 64), -1, np.int32)
    for i, k in enumerate(spec):
        a = int(rng.integers(0, k + 1)) if i != 2 else 63       # (all of them: nothing moves)
        path[i, :a] = np.sort(rng.choice(np.arange(1, k + 1), a, replace=False))
        lens.append(a)
    caches = [cache8(rng, num, hkv, d, loud) for loud in (1.0, 30.0)]
    for x, s in caches:
        s *= 2.0 ** rng.integers(-6, 7, s.shape)                # pages of very different scales
    dp, ds = [dev(x, "e4m3") for x, _ in caches], [dev(s) for _, s in caches]
    pkg.kv_compact_path(*dp, dev(bt), ints(*ctx), ints(*spec), dev(path), ints(*lens), max_spec_len=63, k_scales=ds[0], v_scales=ds[1])
    torch.cuda.synchronize()
    for (x, s), dx, dsx in zip(caches, dp, ds):
        want, want_s = P.compact_path_scaled(x, s, bt, ctx, spec, path, lens)
        assert np.array_equal(host(dsx), want_s.astype(np.float32))
        got = host(dx, "e4m3")
        # rows that are kept: what is behind the last accepted one is dead
        live = np.ones(got.shape[:1] + got.shape[2:3], bool)
        for i, (L, k, a) in enumerate(zip(ctx, spec, lens)):
            for t in range(L - k + a, -(-L // 16) * 16):
                live[bt[i, t // 16], t % 16] = False
        assert np.array_equal(got.transpose(0, 2, 1, 3)[live], want.transpose(0, 2, 1, 3)[live])


def test_paths_that_are_none(pkg):  # noqa: F811
    """Entries that do not rise, or lead outside the request, end the path; requests whose lengths make no sense are left alone."""
    import torch
    rng = np.random.default_rng(5)
    ctx, spec = [40, 40, 3, 40], [5, 5, 5, 5]
    bt, num = table(rng, [40, 40, 40, 40])
    x, s = cache8(rng, num, 2, 64)
    path = np.array([[2, 2, 3, -1, -1, -1], [1, 9, 2, -1, -1, -1], [2, 3, -1, -1, -1, -1], [2, 4, -1, -1, -1, -1]], np.int32)
    bt[3, 2] = num + 5
    dx, ds = [dev(x, "e4m3") for _ in range(2)], [dev(s) for _ in range(2)]
    pkg.kv_compact_path(*dx, dev(bt), ints(*ctx), ints(*spec), dev(path), ints(3, 3, 2, 2), max_spec_len=5, k_scales=ds[0], v_scales=ds[1])
    torch.cuda.synchronize()
    want, want_s = P.compact_path_scaled(x, s, bt[:2], [40, 40], [5, 5], path[:2], [1, 1])
    got = host(dx[0], "e4m3")
    for i in (0, 1):
        for t in range(36):
            assert np.array_equal(got[bt[i, t // 16], :, t % 16], want[bt[i, t // 16], :, t % 16])
    rest = np.setdiff1d(np.arange(num), bt[:2].reshape(-1))
    assert np.array_equal(got[rest], x[rest]) and np.array_equal(host(ds[0])[rest], s[rest])
