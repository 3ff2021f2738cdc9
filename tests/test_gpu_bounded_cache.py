"""A cache that stays bounded, all of it together: steps of a continuous batch whose pages are handed out, forked, given back
behind a window and compacted on the device, with the K/V of two layers, and windowed attention over them at every step
against the formula on the histories kept on the host."""
import numpy as np
import pytest

from oracle.pages import refs_of
from oracle.window import visible
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("f16", 4, 2, 64), ("f32", 2, 1, 64)])
def test_steps_of_a_bounded_cache(dtype, hq, hkv, d, pkg):  # noqa: F811
    import torch
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(hq)
    gen = torch.Generator(device="cuda").manual_seed(d)
    window, sinks, width, NP, layers, most = 40, 5, 40, 80, 2, 4
    half_step = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    pools = [torch.full((layers, NP, hkv, 16, d), float("nan"), dtype=kind, device="cuda") for _ in range(2)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda").reshape(-1)             # noqa: E731
    table, refs = torch.full((0, width), -1, dtype=torch.int32, device="cuda"), torch.zeros(NP, dtype=torch.int32, device="cuda")
    hist = []                                       # per request and layer: K, V rows of its committed tokens, on the host
    committed = ints([])
    longest = forks = moved = 0
    for turn in range(40):
        # who goes on: requests end, fork and change places, new ones start with a prompt
        old = len(hist)
        sources = [s for s in r.permutation(old).tolist() if r.random() < 0.97]
        if sources and len(sources) < 5 and r.random() < 0.6:
            sources += [int(r.choice(sources))] * int(r.integers(1, 3))
        while len(sources) < 3:
            sources.append(-1)
        r.shuffle(sources)
        lens = committed.tolist()
        hist = [[(k.copy(), v.copy()) for k, v in hist[s]] if s >= 0 else [(np.zeros((0, hkv, d)),) * 2] * layers for s in sources]
        have = [lens[s] if s >= 0 else 0 for s in sources]
        n = [int(r.integers(1, most + 1)) if h else int(r.integers(1, 110)) for h in have]
        ctx = [h + x for h, x in zip(have, n)]
        if max(ctx) > width * 16 - 60:
            break
        table, refs, src, dst, status = pkg.kv_remap(table, refs, ints(sources), committed, ints(ctx), window=window, sinks=sinks)
        pkg.kv_copy_pages(*pools, src, dst)
        assert status.tolist()[1] == 0
        forks += int((src >= 0).sum())
        if turn % 3 == 2:                           # as if the pool's end were to be given away: nothing may notice
            table, refs, _, src, dst, status = pkg.kv_compact_pages(table, refs, out_table=table, out_refs=refs)
            pkg.kv_copy_pages(*pools, src, dst)
            moved += int((src >= 0).sum())
            pools[0][:, status.tolist()[0]:] = float("nan")
            pools[1][:, status.tolist()[0]:] = float("nan")
        assert np.array_equal(refs.cpu().numpy(), refs_of(table.cpu().numpy(), NP))
        spec, ctx_d = ints([x - 1 for x in n]), ints(ctx)
        TQ, bound = sum(n), max(n) - 1
        for layer in range(layers):
            new = [torch.randn((TQ, hkv, d), generator=gen, device="cuda").to(kind) for _ in range(2)]
            q = torch.randn((TQ, hq, d), generator=gen, device="cuda").to(kind)
            k, v = pools[0][layer], pools[1][layer]
            pkg.kv_append(*new, k, v, table, ctx_d, spec, max_spec_len=bound)
            out = pkg.verify_attn(q, k, v, table, ctx_d, spec, max_spec_len=bound, window=window, sinks=sinks)
            got, qh = out.double().cpu().numpy(), q.double().cpu().numpy()
            nk, nv = (x.double().cpu().numpy() for x in new)
            row = 0
            for i in range(len(n)):
                K, V = (np.concatenate([h, x[row:row + n[i]]]) for h, x in zip(hist[i][layer], (nk, nv)))
                hist[i][layer] = (K, V)
                for j in range(n[i]):
                    t = visible(have[i] + j, window, sinks)
                    for h in range(hq):
                        s = K[t, h // (hq // hkv)] @ qh[row + j, h] / np.sqrt(d)
                        w = np.exp(s - s.max())
                        want = w @ V[t, h // (hq // hkv)] / w.sum()
                        assert (np.abs(got[row + j, h] - want) <= 2e-5 + half_step * np.abs(want)).all(), (turn, layer, i, j, h)
                row += n[i]
        # some of the drafts are accepted
        accepted = [int(r.integers(0, x)) for x in n]
        toks = ints(r.integers(0, 9, len(n) * (bound + 1)).tolist()).view(len(n), bound + 1)
        committed, _, _ = pkg.commit(toks, ints(accepted), spec, ctx_d, max_spec_len=bound)
        assert committed.tolist() == [c - x + 1 + a for c, x, a in zip(ctx, n, accepted)]
        hist = [[(K[:c], V[:c]) for K, V in h] for h, c in zip(hist, committed.tolist())]
        longest = max(longest, max(ctx))
    # pages behind windows, shared pages and moved ones have all occurred
    assert longest > window + sinks + 32 and forks > 0 and moved > 0
