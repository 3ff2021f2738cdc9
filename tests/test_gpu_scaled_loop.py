"""A continuous batch over a cache in 8 bits, all of it together: pages handed out, forked and moved, keys turned and appended,
attention over two layers with one plan, chains and trees of drafts, an accepted path brought together, committed lengths.

What a token's 8 bits may differ from it by: a rounding to e4m3, half a step of 4 bits, 2^-4 of the value, or half of the least
number, 2^-10 of the scale.  A page that gets louder is rounded again by a power of two: exactly, except of what becomes
subnormal, 2^-10 of the new scale each time, and scales at least double each time: less than 2 * 2^-10 of the last one, together.
The fp32 value of a turned key is within 2^-21 (|a| + |b|) of the oracle's (tests/test_gpu_positions.py), before that."""
import numpy as np
import pytest

from oracle import positions as P
from oracle.pages import refs_of
from tests.ragged_rows import HALF_STEP, LEAST, cache8, dev, host, ints, table, widen
from tests.test_gpu_attn_scaled import TOL
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

LAYERS, POOL, WIDTH = 2, 120, 30


def held(pages, scales, table, i, length):
    """(values, scales) [length][Hkv][d], [length][Hkv][1] of a request's first tokens"""
    t = np.arange(length)
    s = scales[table[i, t // 16]].astype(np.float64)[..., None]
    return P.E4M3[pages[table[i, t // 16], :, t % 16]] * s, s


def near(raw, rot, inter, gain):
    """what the fp32 value of a turned entry may be off by"""
    a_at, b_at = P._pairs(rot, inter)
    out, both = np.zeros(raw.shape), 2.0 ** -21 * gain * (np.abs(raw[..., a_at]) + np.abs(raw[..., b_at]))
    out[..., a_at], out[..., b_at] = both, both
    return out


def check_held(k8, ks, v8, vs, table, i, seen, where):
    """the cache's first tokens of request i against seen = (keys, what these may be off by, values)"""
    keys, err, values = seen
    for pages, scales, want, off in ((k8, ks, keys, err), (v8, vs, values, 0.0)):
        got, s = held(host(pages, "e4m3"), host(scales), table, i, len(want))
        tol = off + 2.0 ** -4 * (np.abs(want) + off) + 2.0 ** -9 * s
        assert (np.abs(got - want) <= tol).all(), where + (np.abs(got - want).max(),)


@pytest.mark.parametrize("dtype,hq,hkv,d,rot,inter", [("bf16", 8, 2, 128, 128, False), ("f16", 4, 2, 64, 32, True), ("f32", 2, 1, 96, 96, False)])
def test_steps_of_a_continuous_batch(dtype, hq, hkv, d, rot, inter, pkg):  # noqa: F811
    import torch
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(hq + d)
    gen = torch.Generator(device="cuda").manual_seed(d)
    freq, gain = pkg.rope_frequencies(rot, base=500.0, device="cuda")
    kw = dict(interleaved=inter, attn_factor=gain)
    # nothing that nobody wrote is a number
    pools = [torch.full((LAYERS, POOL, hkv, 16, d), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.full((LAYERS, POOL, hkv), float("nan"), device="cuda") for _ in range(2)]
    both = dict(k_scales=scales[0], v_scales=scales[1])
    bt_d, refs, committed = ints().view(0, WIDTH), torch.zeros(POOL, dtype=torch.int32, device="cuda"), ints()
    hist = []                       # per request and layer: keys (turned), what these may be off by, values of its committed tokens
    forks = moved = taken = louder = 0
    for turn in range(14):
        is_tree = turn % 2 == 1
        old = len(hist)
        sources = [s for s in r.permutation(old).tolist() if r.random() < 0.9]
        if sources and len(sources) < 4 and r.random() < 0.6:
            sources += [int(r.choice(sources))] * 2
        while len(sources) < 3:
            sources.append(-1)
        r.shuffle(sources)
        lens = committed.tolist()
        none = (np.zeros((0, hkv, d)),) * 3
        hist = [list(hist[s]) if s >= 0 else [none] * LAYERS for s in sources]
        have = [lens[s] if s >= 0 else 0 for s in sources]
        most = 33 if is_tree else 6
        n = [int(r.integers(1, most)) if h or is_tree else int(r.integers(1, 100)) for h in have]
        ctx = [h + x for h, x in zip(have, n)]
        if max(ctx) > WIDTH * 16 - 100:
            break
        bt_d, refs, src, dst, status = pkg.kv_remap(bt_d, refs, ints(*sources), committed, ints(*ctx))
        pkg.kv_copy_pages(*pools, src, dst, **both)
        assert status.tolist()[1] == 0
        forks += int((src >= 0).sum())
        if turn % 3 == 2:
            bt_d, refs, _, src, dst, status = pkg.kv_compact_pages(bt_d, refs, out_table=bt_d, out_refs=refs)
            pkg.kv_copy_pages(*pools, src, dst, **both)
            moved += int((src >= 0).sum())
            first = status.tolist()[0]
            for layer in range(LAYERS):
                for x, s in zip(pools, scales):
                    x[layer, first:].view(torch.uint8).fill_(0x7f)
                    s[layer, first:] = float("nan")
        bt = bt_d.cpu().numpy()
        assert np.array_equal(refs.cpu().numpy(), refs_of(bt, POOL))
        B, TQ, bound = len(n), sum(n), max(n) - 1
        spec, ctx_d = ints(*(x - 1 for x in n)), ints(*ctx)
        up = [0 if j == 0 else int(r.integers(max(0, j - 4), j)) for x in n for j in range(x)]
        parents = ints(*up) if is_tree else None
        up = np.array(up) if is_tree else None
        ws = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
        print(f"[case] step {turn} {dtype} B={B} TQ={TQ} tree={is_tree}", flush=True)
        fresh = []
        for layer in range(LAYERS):
            k8, v8, ks, vs = pools[0][layer], pools[1][layer], scales[0][layer], scales[1][layer]
            # queries, keys and values are slices of one product's rows; some steps are louder than others
            rows = torch.randn((TQ, hq + 2 * hkv, d), generator=gen, device="cuda")
            rows[:, hq:] *= 2.0 ** (turn * 5 % 4 - 2)
            rows = rows.to(kind)
            q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
            before = ks.clone()
            turned = pkg.kv_append_rope(q, k, v, freq, k8, v8, bt_d, ctx_d, spec, max_spec_len=bound, k_scales=ks, v_scales=vs, parents=parents, **kw)
            louder += int((ks > before).sum())
            call = dict(max_spec_len=bound, parents=parents, k_scales=ks, v_scales=vs, workspace=ws)
            if layer == 0:
                pkg.verify_attn(turned, k8, v8, bt_d, ctx_d, spec, plan="build", **call)
            out = pkg.verify_attn(turned, k8, v8, bt_d, ctx_d, spec, plan="reuse", out_dtype=0, **call)
            # attention: of what the cache holds (keys are up to twice those that TOL was made for, which scales the scores' error)
            args = [host(turned, dtype), host(k8, "e4m3"), host(v8, "e4m3"), host(ks), host(vs), bt, ctx, [x - 1 for x in n]]
            ref = P.verify_attn_scaled(*args, dtype=dtype, parents=up)
            args[2] = np.where(args[2] & 0x7f == 0x7f, args[2], args[2] & 0x7f)
            size = P.verify_attn_scaled(*args, dtype=dtype, parents=up)
            fast = d in (64, 128) and dtype != "f32"
            off = np.abs(host(out).astype(np.float64) - ref)
            assert (off <= 2 * TOL * max(1.0, size.max()) + (2.0 ** -11 * size if fast else 0.0)).all(), (turn, layer, off.max())
            # queries: of the positions that the rows have
            more = dict(dtype=dtype, interleaved=inter, attn_factor=gain, parents=up)
            raw = [widen(host(x.contiguous(), dtype), dtype) for x in (q, k, v)]
            f = host(freq)
            want = P.rope(host(q.contiguous(), dtype), f, ctx, args[7], **more)
            off = near(raw[0], rot, inter, gain)
            assert (np.abs(widen(args[0], dtype) - want) <= off + HALF_STEP[dtype] * (np.abs(want) + off) + LEAST[dtype]).all()
            # the cache: every token of every request
            key, row = P.rope(host(k.contiguous(), dtype), f, ctx, args[7], **more), 0
            err, new = near(raw[1], rot, inter, gain), []
            for i in range(B):
                part = slice(row, row + n[i])
                seen = [np.concatenate([h, x[part]]) for h, x in zip(hist[i][layer], (key, err, raw[2]))]
                check_held(k8, ks, v8, vs, bt, i, seen, (turn, layer, i))
                new.append(tuple(seen))
                row += n[i]
            fresh.append(new)
        # some of the drafts are accepted, with few tokens to choose from
        V = 7
        logits = torch.randn((TQ, V), generator=gen, device="cuda")
        probs = torch.softmax(torch.randn((TQ - B, V), generator=gen, device="cuda"), dim=1)
        toks = torch.randint(0, V, (TQ - B,), generator=gen, device="cuda", dtype=torch.int32)
        temp = torch.ones(B, device="cuda")
        uni = torch.rand((TQ, 2), generator=gen, device="cuda")
        if is_tree:
            ids, accepted, path = pkg.accept_tree(logits, probs, toks, parents, uni, spec, temp, max_spec_len=bound)
            for layer in range(LAYERS):
                pkg.kv_compact_path(pools[0][layer], pools[1][layer], bt_d, ctx_d, spec, path, accepted, max_spec_len=bound,
                                    k_scales=scales[0][layer], v_scales=scales[1][layer])
            path = path.cpu().numpy()
        else:
            ids, accepted = pkg.accept(logits, probs, toks, uni, spec, temp, max_spec_len=bound)
        committed, _, _ = pkg.commit(ids, accepted, spec, ctx_d, max_spec_len=bound)
        acc = accepted.tolist()
        assert committed.tolist() == [h + 1 + a for h, a in zip(have, acc)]
        taken += sum(acc)
        for i in range(B):
            keep = list(range(have[i] + 1)) + [have[i] + (int(path[i, j]) if is_tree else 1 + j) for j in range(acc[i])]
            hist[i] = [tuple(x[keep] for x in fresh[layer][i]) for layer in range(LAYERS)]
            for layer in range(LAYERS):
                check_held(pools[0][layer], scales[0][layer], pools[1][layer], scales[1][layer], bt, i, hist[i][layer], (turn, layer, i, "kept"))
    assert forks > 0 and moved > 0 and taken > 0 and louder > 0


def test_appends_in_graphs_on_streams_and_in_threads(pkg):  # noqa: F811
    """Two batches' appends with their attention, captured and replayed together with eager ones: no call shares anything with another."""
    import threading
    import torch
    jobs = []
    for n in range(2):
        rng = np.random.default_rng(60 + n)
        B, hq, hkv, d = (130, 20)[n], 8, 2, (64, 128)[n]
        spec = [int(x) for x in rng.integers(0, 7, B)]
        ctx = [int(x) + k + 1 for x, k in zip(rng.integers(0, 400, B), spec)]
        bt, num = table(rng, ctx)
        TQ = sum(spec) + B
        start = [*cache8(rng, num, hkv, d), *cache8(rng, num, hkv, d, 0.3)]
        start = [dev(x, "e4m3" if i % 2 == 0 else None) for i, x in enumerate(start)]
        rows = [torch.randn((TQ, h, d), device="cuda").bfloat16() for h in (hq, hkv, hkv)]
        ints_ = (dev(bt), ints(*ctx), ints(*spec))
        freq = pkg.rope_frequencies(d, device="cuda")[0]

        def run(c, rows=rows, ints_=ints_, freq=freq, stream=None):
            kw = dict(max_spec_len=6, k_scales=c[1], v_scales=c[3], stream=stream)
            q = pkg.kv_append_rope(*rows, freq, c[0], c[2], *ints_, **kw)
            c.append(q)                 # (a new tensor of the current stream: it has to stay until `stream` has used it)
            return pkg.verify_attn(q, c[0], c[2], *ints_, **kw)
        first = [x.clone() for x in start]
        jobs.append((run, start, first, run(first)))
    torch.cuda.synchronize()

    def same(c, out, want, want_out):
        return torch.equal(out, want_out) and all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(c, want))
    graphs = []
    for run, start, _, _ in jobs:
        c = [x.clone() for x in start]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run(c)
        graphs.append((g, c, out))
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        for (g, c, out), (_, start, _, _) in zip(graphs, jobs):
            out.zero_()
            for x, y in zip(c, start):
                x.copy_(y)
            c[4].zero_()
        eager = [[x.clone() for x in start] for _, start, _, _ in jobs]
        torch.cuda.synchronize()
        for (g, _, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        outs = [run(c, stream=s) for (run, _, _, _), c, s in zip(jobs, eager, streams[::-1])]
        torch.cuda.synchronize()
        for (g, c, out), e, o, (_, _, want, want_out) in zip(graphs, eager, outs, jobs):
            assert same(c, out, want, want_out) and same(e, o, want, want_out)
    results = [[] for _ in jobs]

    def work(i):
        run, start, _, _ = jobs[i]
        with torch.cuda.stream(streams[i]):
            for _ in range(8):
                c = [x.clone() for x in start]
                results[i].append((c, run(c)))
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    for got, (_, _, want, want_out) in zip(results, jobs):
        assert len(got) == 8 and all(same(c, out, want, want_out) for c, out in got)
