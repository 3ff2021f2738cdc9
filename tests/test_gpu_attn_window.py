"""Windowed verification attention (csrc/attn_window*.hip) against the oracle in 64 bits.

Everything that a row must not see is poisoned: tokens that no row of a request sees hold NaN, pages made of such tokens
have no entry in the block table (-1), unused slots hold NaN (the workload's own).

Tolerance on the fp32 accumulator: that of the other attention tests, 2e-5.  Scores, weights and sums are fp32; the matrix cores
take 16-bit weights in two pieces, which leave 2^-24 (f16) or 2^-18 (bf16) of a weight out: of a mean of values below 5, 1.9e-5 if
every weight were off by that much to the same side.  16-bit outputs: half a step of the type on top, 2^-9 (bf16) or 2^-12
(fp16) of the next power of two above the value, which is at most 2^-8 or 2^-11 of the value."""
import numpy as np
import pytest

import workloads as W
from oracle.window import hidden_tokens, verify_attn_window
from tests.harness import to_device
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def poisoned(st, window, sinks, holes=True):
    """What no row sees: NaN in the cache, no page in the table (`holes`)."""
    nan = np.uint16(0x7FC0) if st.dtype == "bf16" else np.nan
    for i in range(st.batch):
        t = hidden_tokens(int(st.ctx_lens[i]), int(st.spec_lens[i]) + 1, window, sinks)
        for pages in (st.k_pages, st.v_pages):
            pages[st.block_table[i, t // 16], :, t % 16] = nan
        if holes:
            p, n = np.unique(t // 16, return_counts=True)
            st.block_table[i, p[n == 16]] = -1
    return st


def run(pkg, st, window, sinks, **kw):  # noqa: F811
    import torch
    d = to_device(st, acceptance=False)
    out = torch.full(st.q.shape, float("nan"), device="cuda", dtype=torch.float32 if kw.get("out_dtype") == 0 else d.q.dtype)
    r = pkg.verify_attn(d.q, d.k_pages, d.v_pages, d.block_table, d.ctx_lens, d.spec_lens, out, max_spec_len=kw.pop("max_spec_len", st.max_spec_len),
                        window=window, sinks=sinks, **kw)
    torch.cuda.synchronize()
    assert r is out
    return out.double().cpu().numpy()


def check(pkg, st, window, sinks, paths=("auto", "vector")):  # noqa: F811
    ref = verify_attn_window(st.q, st.k_pages, st.v_pages, st.block_table, st.ctx_lens, st.spec_lens, window=window, sinks=sinks,
                             dtype=st.dtype)
    for path in paths:
        print(f"[case] {st.name} {st.dtype} d={st.head_dim} {st.n_q_heads}/{st.n_kv_heads} B={st.batch} window={window} sinks={sinks} {path}", flush=True)
        out = run(pkg, st, window, sinks, out_dtype=0, path=path)
        err = np.abs(out - ref)
        assert not np.isnan(out).any() and err.max() <= 2e-5, (path, err.max())
        own = run(pkg, st, window, sinks, path=path)
        assert (np.abs(own - ref) <= 2e-5 + HALF_STEP[st.dtype] * np.abs(ref)).all(), path


def step(seed, ctx, spec, hq, hkv, d, dtype, name="window"):
    return W.make_custom_step(seed, ctx_lens=ctx, spec_lens=spec, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=dtype,
                              acceptance=False, name=name)


SHAPES = [
    # ctx_lens, spec_lens, Hq, Hkv
    ([1, 2, 16, 17, 31, 33, 64, 65], [0, 1, 0, 2, 1, 3, 0, 4], 2, 2),
    ([140, 257, 300, 19, 512, 1030], [3, 0, 5, 1, 8, 2], 8, 2),              # up to 36 rows a kv head
    ([90, 700, 33], [10, 12, 0], 16, 2),                                      # G = 8: 104 rows, two row groups
    ([400, 5, 90], [7, 3, 0], 14, 2),                                         # G = 7
]
WINDOWS = [(1, 0), (1, 1), (7, 0), (16, 4), (17, 16), (32, 33), (100, 3), (129, 0), (1000, 20), (4096, 0), ((1 << 31) - 1, 0)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{len(s[0])}-L{max(s[0])}-k{max(s[1])}-{s[2]}x{s[3]}")
def test_windows_and_sinks(shape, d, dtype, pkg):  # noqa: F811
    ctx, spec, hq, hkv = shape
    for window, sinks in WINDOWS:
        check(pkg, poisoned(step(900 + d, ctx, spec, hq, hkv, d, dtype), window, sinks), window, sinks)


@pytest.mark.parametrize("d,dtype", [(8, "bf16"), (40, "f32"), (80, "f16"), (96, "bf16"), (192, "f16"), (256, "f32")])
def test_other_head_dims(d, dtype, pkg):  # noqa: F811
    for window, sinks in ((5, 2), (64, 0), (150, 17)):
        st = poisoned(step(950 + d, [3, 90, 260, 33], [1, 6, 0, 2], 6, 2, d, dtype), window, sinks)
        check(pkg, st, window, sinks, paths=("auto",))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 64)])
def test_long_contexts_and_few_pairs(dtype, d, pkg):  # noqa: F811
    """One request, one kv head: units cut into parts that are merged."""
    for window, sinks in ((4096, 4), (2047, 70), (6000, 0), (700, 1)):
        check(pkg, poisoned(step(970, [9000], [4], 4, 1, d, dtype), window, sinks), window, sinks, paths=("auto",))
    check(pkg, poisoned(step(971, [5000, 64, 3000], [2, 3, 0], 4, 2, d, dtype), 2500, 8), 2500, 8, paths=("auto",))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_many_units(dtype, d, pkg):  # noqa: F811
    rng = np.random.default_rng(5)
    ctx, spec = rng.integers(9, 400, 150), rng.integers(0, 7, 150)
    check(pkg, poisoned(step(980, ctx.tolist(), spec.tolist(), 8, 4, d, dtype), 77, 5), 77, 5, paths=("auto",))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 128), ("f32", 64), ("bf16", 64)])
def test_long_drafts(dtype, d, pkg):  # noqa: F811
    """Hundreds of query rows beside single ones: every row group has a window of its own."""
    for window, sinks in ((40, 3), (300, 0)):
        check(pkg, poisoned(step(990, [333, 700, 20], [299, 0, 19], 4, 2, d, dtype), window, sinks), window, sinks, paths=("auto",))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("path", ["auto", "vector"])
def test_what_a_row_does_not_see_cannot_reach_it(dtype, path, pkg):  # noqa: F811
    """NaN and infinities in tokens that some rows of a request see and others do not.  Rows that see none of them are worked
out in another way than without them: both are fp32 (2e-6), but the matrix cores take bf16 weights in two pieces, of which the
first is off by at most 2^-9 of the weight and the second by at most 2^-9 of that: 2^-18 of a mean of values below 5."""
    window, sinks = 20, 2
    tol = 2e-6 + (5 * 2.0 ** -18 if dtype == "bf16" else 0.0)
    for d in (64, 128):
        for bad in (np.nan, np.inf, -np.inf):
            st = step(1000, [50, 90], [5, 7], 8, 2, d, dtype)
            bits = {np.inf: 0x7F80, -np.inf: 0xFF80}.get(bad, 0x7FC0)
            bad_bits = np.uint16(bits) if dtype == "bf16" else bad
            clean = run(pkg, st, window, sinks, out_dtype=0, path=path)
            for i in range(2):
                L, n = int(st.ctx_lens[i]), int(st.spec_lens[i]) + 1
                for t in (L - n - window + 3, L - 2):               # out of the later rows' windows; a draft that the last two rows see
                    st.v_pages[st.block_table[i, t // 16], :, t % 16, 1::3] = bad_bits
                    st.k_pages[st.block_table[i, t // 16], :, t % 16, 5] = bad_bits
            out = run(pkg, st, window, sinks, out_dtype=0, path=path)
            row = 0
            for i in range(2):
                L, n = int(st.ctx_lens[i]), int(st.spec_lens[i]) + 1
                for j in range(n):
                    pos = L - n + j
                    if any(t <= pos and pos - t < window for t in (L - n - window + 3, L - 2)):
                        assert not np.isfinite(out[row]).all(), (d, bad, i, j)
                    else:
                        assert float(np.abs(out[row] - clean[row]).max()) <= tol, (d, bad, i, j)
                    row += 1


def test_scores_of_any_size(pkg):  # noqa: F811
    import torch
    for dtype, size in (("f32", 1e15), ("bf16", 1e15), ("f16", 200.0)):
        for d in (64, 128):
            st = step(1010, [200, 40], [3, 1], 4, 2, d, dtype)
            s = to_device(st, acceptance=False)
            q, k = (s.q.float() * size).to(s.q.dtype), (s.k_pages.float() * size).to(s.q.dtype)
            out = pkg.verify_attn(q, k, s.v_pages, s.block_table, s.ctx_lens, s.spec_lens, max_spec_len=3, window=60, sinks=3, out_dtype=0)
            assert torch.isfinite(out).all()
            # the weight of one token dominates: the output is a row of V
            row = out[0, 0]
            page = s.block_table[0, :13].long()
            rows = s.v_pages[page, 0].float().reshape(-1, d)
            rows = rows[torch.isfinite(rows).all(dim=1)]
            assert (rows - row).abs().amax(dim=1).min() <= 2e-5


def test_scale_strides_and_bounds(pkg):  # noqa: F811
    st = poisoned(step(1020, [64, 200, 30], [2, 4, 0], 8, 2, 128, "bf16"), 50, 4)
    for scale in (0.02, 1.0):
        ref = verify_attn_window(st.q, st.k_pages, st.v_pages, st.block_table, st.ctx_lens, st.spec_lens, window=50, sinks=4, dtype="bf16",
                                 scale=scale)
        out = run(pkg, st, 50, 4, out_dtype=0, scale=scale, max_spec_len=9)             # a bound above the longest
        assert np.abs(out - ref).max() <= 2e-5


def test_plans_streams_workspaces_and_repeats(pkg):  # noqa: F811
    import torch
    st = poisoned(step(1030, [3000, 41, 700], [4, 0, 2], 8, 2, 128, "bf16"), 1500, 4)
    d = to_device(st, acceptance=False)
    args = (d.q, d.k_pages, d.v_pages, d.block_table, d.ctx_lens, d.spec_lens)
    kw = dict(max_spec_len=4, window=1500, sinks=4)
    ref = pkg.verify_attn(*args, **kw)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda").random_(0, 256)
    assert pkg.verify_attn(*args, plan="build", workspace=ws, **kw) is None
    for _ in range(3):
        ws.random_(0, 256)                                          # nothing in it is relied on
        assert torch.equal(pkg.verify_attn(*args, plan="reuse", workspace=ws, **kw), ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = pkg.verify_attn(*args, workspace=ws, **kw)
    side.synchronize()
    assert torch.equal(out, ref)


def test_captured_and_replayed(pkg):  # noqa: F811
    """Two captured calls that share a workspace, replayed between eager calls of other sizes in the same workspace."""
    import torch
    st = poisoned(step(1040, [3000, 41, 700], [4, 0, 2], 8, 2, 128, "bf16"), 1500, 4)
    d = to_device(st, acceptance=False)
    args = (d.k_pages, d.v_pages, d.block_table, d.ctx_lens, d.spec_lens)
    kw = dict(max_spec_len=4, window=1500, sinks=4)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    qs = [d.q.clone(), d.q.flip(0).contiguous()]
    outs = [torch.empty_like(d.q) for _ in qs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for q, o in zip(qs, outs):
            pkg.verify_attn(q, *args, o, workspace=ws, **kw)
    side.synchronize()
    for q, o in zip(qs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            pkg.verify_attn(q, *args, o, workspace=ws, **kw)
        graphs.append(g)
    torch.cuda.synchronize()
    gen = torch.Generator(device="cuda")
    for k in range(4):
        for q in qs:
            q.copy_(torch.randn(q.shape, generator=gen.manual_seed(k), device="cuda"))
        torch.cuda.synchronize()
        for g, q, o in zip(graphs, qs, outs):
            g.replay()
            pkg.verify_attn(q, *args, workspace=ws, max_spec_len=4, window=900, sinks=0, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        for q, o in zip(qs, outs):
            assert torch.equal(o, pkg.verify_attn(q, *args, **kw))


def test_checked_inputs(pkg):  # noqa: F811
    """The device-side check leaves out what a windowed call never reads."""
    st = poisoned(step(1050, [300, 41], [4, 0], 8, 2, 128, "bf16"), 50, 4)
    d = to_device(st, acceptance=False)
    dims = pkg.attn_dims(d.q, d.k_pages, d.block_table, max_spec_len=4)
    assert (st.block_table[0, :19] < 0).any()
    assert pkg.check_ragged_inputs(d.block_table, d.ctx_lens, d.spec_lens, dims) == 4
    assert pkg.check_ragged_inputs(d.block_table, d.ctx_lens, d.spec_lens, dims, window=50, sinks=4) == 0
    assert pkg.check_ragged_inputs(d.block_table, d.ctx_lens, d.spec_lens, dims, window=50, sinks=20) == 4
    assert pkg.check_ragged_inputs(d.block_table, d.ctx_lens, d.spec_lens, dims, window=90, sinks=4) == 4
