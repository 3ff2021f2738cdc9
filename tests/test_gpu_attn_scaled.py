"""Verification attention over the cache in 8 bits (csrc/attn_e4m3.hip, attn_vector.hip) against the oracle in 64 bits.

Tolerance on the fp32 accumulator: 2e-5 for values of unit size, that of the other attention tests, where weights are fp32 (the
portable form).  On the matrix cores keys and values are exact in the products, the softmax weights are f16: each is off by up to half
a step of 11 bits, torch.finfo(torch.float16).eps / 2 = 2^-11 of it, and a mean of values by up to 2^-11 times the mean of their magnitudes, which the oracle's weights give row by
row and channel by channel.  Outputs of 16 bits: half a step on top."""
import numpy as np
import pytest

from oracle import positions as P
from tests.ragged_rows import HALF_STEP, LEAST, cache8, dev, host, ints, store, table, tree, widen
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

TOL = 2e-5


def make(seed, ctx, spec, hq, hkv, d, dtype, is_tree=False, width=None):
    rng = np.random.default_rng(seed)
    bt, num = table(rng, ctx, width=width)
    (k8, ks), (v8, vs) = cache8(rng, num, hkv, d), cache8(rng, num, hkv, d)
    k8, v8 = k8.copy(), v8.copy()
    # scales that are no powers of two, and slots and pages that nobody uses: NaN
    ks, vs = (ks * rng.uniform(0.7, 1.0, ks.shape)).astype(np.float32), (vs * rng.uniform(0.7, 1.0, vs.shape)).astype(np.float32)
    used = np.zeros(num, bool)
    for i, L in enumerate(ctx):
        used[bt[i, :-(-L // 16)]] = True
        if L % 16:
            k8[bt[i, L // 16], :, L % 16:], v8[bt[i, L // 16], :, L % 16:] = 0x7f, 0xff
    ks[~used], vs[~used] = np.nan, np.nan
    TQ = sum(spec) + len(spec)
    return dict(q=store(rng.normal(0, 1, (TQ, hq, d)), dtype), k8=k8, v8=v8, ks=ks, vs=vs, bt=bt, ctx=ctx, spec=spec, dtype=dtype,
                parents=tree(rng, spec) if is_tree else None)


def call(pkg, c, **kw):  # noqa: F811
    import torch
    kw.setdefault("max_spec_len", max(c["spec"]))
    out = pkg.verify_attn(dev(c["q"], c["dtype"]), dev(c["k8"], "e4m3"), dev(c["v8"], "e4m3"), dev(c["bt"]), ints(*c["ctx"]), ints(*c["spec"]),
                          k_scales=dev(c["ks"]), v_scales=dev(c["vs"]), parents=None if c["parents"] is None else dev(c["parents"]), **kw)
    torch.cuda.synchronize()
    return out


def oracle(c):
    """(outputs, the mean of the values' magnitudes with the same weights)"""
    magnitudes = dict(c, v8=np.where(c["v8"] & 0x7f == 0x7f, c["v8"], c["v8"] & 0x7f))
    return _oracle(c), _oracle(magnitudes)


def _oracle(c):
    return P.verify_attn_scaled(c["q"], c["k8"], c["v8"], c["ks"], c["vs"], c["bt"], c["ctx"], c["spec"], dtype=c["dtype"], parents=c["parents"])


def check(pkg, c, paths=("auto", "vector"), ref=None, **kw):  # noqa: F811
    ref, size = oracle(c) if ref is None else ref
    fast = c["q"].shape[2] in (64, 128) and c["dtype"] != "f32"
    for path in paths:
        tol = TOL + (2.0 ** -11 * size if fast and path == "auto" else 0.0) + np.zeros(ref.shape)
        print(f"[case] attn8 {c['dtype']} {c['q'].shape} Hkv={c['k8'].shape[1]} B={len(c['ctx'])} tree={c['parents'] is not None} {path}", flush=True)
        out = host(call(pkg, c, out_dtype=0, path=path, **kw)).astype(np.float64)
        assert np.array_equal(np.isnan(out), np.isnan(ref)), path
        fine = ~np.isnan(ref)
        assert (np.abs(out - ref) <= tol)[fine].all(), (path, np.abs(out - ref)[fine].max())
        own = widen(host(call(pkg, c, path=path, **kw), c["dtype"]), c["dtype"])
        tol = tol + HALF_STEP[c["dtype"]] * (np.abs(ref) + tol) + LEAST[c["dtype"]]
        assert (np.abs(own - ref) <= tol)[fine].all(), path


SHAPES = [
    # ctx_lens, spec_lens, Hq, Hkv
    ([1, 2, 16, 17, 31, 33, 64, 65, 63, 32], [0, 1, 0, 2, 1, 3, 0, 4, 0, 0], 2, 2),
    ([140, 257, 300, 19, 512, 1030], [3, 0, 5, 1, 7, 2], 8, 2),             # up to 32 rows a kv head
    ([90, 700, 33], [10, 11, 0], 8, 2),                                      # 48 rows
    ([90, 700, 33], [10, 12, 0], 16, 2),                                     # G = 8: 104 rows, two row groups
    ([400, 5, 90], [7, 3, 0], 14, 2),                                        # G = 7: 56 rows
    ([64, 333], [63, 40], 3, 3),                                             # all of a context is new
]


@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (64, "bf16"), (64, "f32"), (128, "f16"), (128, "bf16"), (128, "f32"), (96, "bf16"), (256, "bf16")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{len(s[0])}-L{max(s[0])}-k{max(s[1])}-{s[2]}x{s[3]}")
def test_shapes(shape, d, dtype, is_tree, pkg):  # noqa: F811
    ctx, spec, hq, hkv = shape
    check(pkg, make(40 + d, ctx, spec, hq, hkv, d, dtype, is_tree), paths=("auto", "vector") if d in (64, 128) and dtype != "f32" else ("auto",))


@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("width", [None, 600, 4000])
def test_splits(width, d, is_tree, pkg):  # noqa: F811
    """Tables of several widths: direct calls, merged or combined splits, scheduled calls of one or several splits."""
    for n, (ctx, spec, hq, hkv) in enumerate([([5000], [5], 8, 2), ([5000, 1, 300, 2049, 2048], [5, 0, 3, 7, 1], 16, 4), ([700, 2100, 513], [2, 30, 0], 4, 2)]):
        check(pkg, make(7 + n, ctx, spec, hq, hkv, d, "bf16", is_tree, width), paths=("auto",))


def test_many_requests(pkg):  # noqa: F811
    rng = np.random.default_rng(11)
    for d, hq, hkv, B in ((128, 4, 2, 300), (64, 8, 8, 150), (128, 8, 1, 1100)):
        ctx = [int(x) for x in rng.integers(8, 400 if B < 1000 else 40, B)]
        check(pkg, make(B, ctx, [int(x) for x in rng.integers(0, 8, B)], hq, hkv, d, "f16"), paths=("auto",))


@pytest.mark.parametrize("d", [64, 128, 96])
@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
def test_a_token_counts_only_where_it_is_seen(is_tree, d, pkg):  # noqa: F811
    """NaN keys, values and scales of drafts: rows that see them are NaN (a value: in its channels), the others as if it were not there."""
    ctx, spec = [200, 77, 40, 31], [9, 12, 3, 0]
    for what in ("key", "value", "value on a page border", "scales"):
        c = make(3, ctx, spec, 8, 2, d, "bf16", is_tree)
        for i, t in ((0, 195), (1, 70), (2, 38)):
            page, slot = c["bt"][i, t // 16], t % 16
            if what == "key":
                c["k8"][page, 1, slot, 5] = 0x7f
            elif what == "value":
                c["v8"][page, 0, slot, [3, d - 1]] = 0xff
            elif what == "value on a page border":
                page, slot = c["bt"][i, (ctx[i] - 1) // 16], (ctx[i] - 1) % 16
                c["v8"][page, :, slot, d // 2] = 0x7f
            elif t // 16 == (ctx[i] - 1) // 16 and (ctx[i] - spec[i] - 1) // 16 < t // 16:
                c["vs"][page, 0] = np.nan                   # a page of drafts alone
        ref = oracle(c)
        if what != "scales":
            assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
        check(pkg, c, ref=ref)


def test_keys_that_are_all_nan_or_zero(pkg):  # noqa: F811
    c = make(9, [100, 40], [4, 2], 4, 2, 128, "f16")
    c["k8"][c["bt"][0, :7]] = 0                              # scores all equal: the mean of the values
    c["k8"][c["bt"][1, 0], 0] = 0x7f
    check(pkg, c)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_large_scores_and_scales(dtype, pkg):  # noqa: F811
    """Scores of thousands, values of 2^40: differences of scores decide, and nothing overflows on the way.  Scores below 2^13 are off
    by 2^-10 at most, a weight by 0.1 % then; values relative to their scale."""
    c = make(12, [300, 33], [5, 0], 8, 2, 128, dtype)
    c["ks"] *= np.float32(400.0)
    c["vs"] *= np.float32(2.0 ** 40)
    ref, _ = oracle(c)
    for path in ("auto", "vector"):
        out = host(call(pkg, c, out_dtype=0, path=path)).astype(np.float64)
        assert np.abs(out - ref).max() <= 4e-3 * 2.0 ** 40 * 5


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("apart", [4, 9, 20, 60, -30])
def test_pages_of_very_different_scales(apart, is_tree, d, pkg):  # noqa: F811
    """Single pages 2^apart as loud as the others, whose weights are as much smaller, or the square of that, or hidden from most rows.

    Tolerance, relative to the mean of the values' magnitudes under the exact weights: 2^-11 for the f16 weights (as above); fp32 scores of up to
    `most` in magnitude are sums of d products and two factors, off by (d + 2) 2^-24 of it, weights and their sum by that much each; TOL for
    the rest.  What is lost to f16 subnormals: 2^-26 of the row's largest weighted scale per token."""
    ctx, spec = [593, 900, 2100, 33], [6, 5, 3, 1]          # (593, 33: the last token is alone in its page, and hidden from the other rows)
    for square in (1, 2):
        c = make(40 + square, ctx, spec, 8, 2, d, "bf16", is_tree)
        c["q"] = store(np.abs(widen(c["q"], "bf16")), "bf16")
        for i, L in enumerate(ctx):
            loud = {L // 64, (L - 1) // 16 - 9, (L - 1) // 16} if L > 200 else {(L - 1) // 16}
            for p in loud:
                page = c["bt"][i, p]
                c["vs"][page] *= np.float32(2.0 ** apart)
                if p < (L - 1) // 16:                       # scores of about -apart * square, in log2, everywhere in it
                    c["k8"][page] = P.to_e4m3(np.array([-256.0]))[0]
                    c["ks"][page] = max(apart, 0) * square * np.log(2.0) / (0.8 * np.sqrt(d)) / 256.0
        ref, size = oracle(c)
        k = P.E4M3[c["k8"]] * c["ks"][..., None, None].astype(np.float64)
        longest = np.sqrt(np.nanmax((np.nan_to_num(k) ** 2).sum(-1)) * (widen(c["q"], "bf16") ** 2).sum(-1).max()) / np.sqrt(d)
        tol = (TOL + 2.0 ** -11 + 2 * (d + 2) * 2.0 ** -24 * longest) * size + 2.0 ** -26 * max(ctx) * size.max(axis=-1, keepdims=True)
        for path in ("auto", "vector"):
            off = np.abs(host(call(pkg, c, out_dtype=0, path=path)).astype(np.float64) - ref)
            assert (off <= tol).all(), (square, path, (off / size).max())


def test_plans_graphs_streams_and_threads(pkg):  # noqa: F811
    import threading
    import torch
    jobs = []
    for n, is_tree in enumerate((False, True, False)):
        rng = np.random.default_rng(20 + n)
        ctx = [int(x) for x in rng.integers(70, 3000, 40)]
        c = make(30 + n, ctx, [int(x) for x in rng.integers(0, 7, 40)], 8, 2, (128, 64, 128)[n], "bf16", is_tree)
        t = [dev(c["q"], "bf16"), dev(c["k8"], "e4m3"), dev(c["v8"], "e4m3"), dev(c["bt"]), ints(*c["ctx"]), ints(*c["spec"])]
        kw = dict(max_spec_len=6, k_scales=dev(c["ks"]), v_scales=dev(c["vs"]), parents=None if c["parents"] is None else dev(c["parents"]))
        want = pkg.verify_attn(*t, **kw)
        ref, size = oracle(c)
        tol = TOL + 2.0 ** -11 * size
        assert (np.abs(widen(host(want, "bf16"), "bf16") - ref) <= tol + HALF_STEP["bf16"] * (np.abs(ref) + tol)).all()
        jobs.append((t, kw, want))
        # metadata once, then used
        ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        assert pkg.verify_attn(*t, plan="build", workspace=ws, **kw) is None
        for _ in range(2):
            assert torch.equal(pkg.verify_attn(*t, plan="reuse", workspace=ws, **kw), want)
    graphs = []
    for t, kw, want in jobs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = pkg.verify_attn(*t, **kw)
        graphs.append((g, out, want))
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        for g, out, _ in graphs:
            out.zero_()
        torch.cuda.synchronize()
        for (g, _, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = [pkg.verify_attn(*t, stream=s, **kw) for (t, kw, _), s in zip(jobs, streams)]
        torch.cuda.synchronize()
        for (_, out, want), e in zip(graphs, eager):
            assert torch.equal(out, want) and torch.equal(e, want)
    results = [None] * len(jobs)

    def work(i):
        with torch.cuda.stream(streams[i]):
            results[i] = [pkg.verify_attn(*jobs[i][0], **jobs[i][1]) for _ in range(10)]
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    for r, (_, _, want) in zip(results, jobs):
        assert all(torch.equal(x, want) for x in r)


def test_a_pool_beyond_32_bits(pkg):  # noqa: F811
    """Pages whose bytes lie behind 2^32."""
    import torch
    hkv, d, num = 8, 128, 280000                            # 4.6 GB of K
    k8, v8 = (torch.zeros((num, hkv, 16, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((num, hkv), device="cuda") for _ in range(2))
    c = make(77, [100, 50], [3, 1], 16, hkv, d, "bf16")
    far = np.arange(num - len(c["ks"]), num)
    for t, x in ((k8, c["k8"]), (v8, c["v8"])):
        t[num - len(x):] = torch.from_numpy(x).cuda()
    for t, x in ((ks, c["ks"]), (vs, c["vs"])):
        t[num - len(x):] = torch.from_numpy(x).cuda()
    bt = np.where(c["bt"] >= 0, far[np.maximum(c["bt"], 0)], -1).astype(np.int32)
    (ref, size), e8 = oracle(c), torch.float8_e4m3fn
    for path in ("auto", "vector"):
        out = pkg.verify_attn(dev(c["q"], "bf16"), k8.view(e8), v8.view(e8), dev(bt), ints(100, 50), ints(3, 1), max_spec_len=3, k_scales=ks, v_scales=vs,
                              out_dtype=0, path=path)
        assert (np.abs(host(out) - ref) <= TOL + 2.0 ** -11 * size).all()
    # an append there
    kn, vn = (torch.randn((6, hkv, d), device="cuda").bfloat16() for _ in range(2))
    pkg.kv_append(kn, vn, k8.view(e8), v8.view(e8), dev(bt), ints(100, 50), ints(3, 1), max_spec_len=3, k_scales=ks, v_scales=vs)
    wk, wv, wks, wvs = P.append_scaled(host(kn, "bf16"), host(vn, "bf16"), None, c["k8"], c["v8"], c["ks"], c["vs"], c["bt"], [100, 50], [3, 1], dtype="bf16")
    assert np.array_equal(host(k8[num - len(wk):]), wk) and np.array_equal(host(v8[num - len(wv):]), wv)
    assert np.array_equal(host(ks[num - len(wk):]), wks.astype(np.float32), equal_nan=True)
