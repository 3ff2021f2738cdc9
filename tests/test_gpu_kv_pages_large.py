"""Remap and compaction of large batches and pools, at the limits between their forms, captured, and from two streams at once;
against the oracle: integers, so everything is equal."""
import numpy as np
import pytest

from oracle.pages import kv_compact_pages, kv_remap, refs_of
from tests.test_gpu_kv_pages import check_compact, check_remap, dev, state
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("old,B,width,slack", [(1024, 1024, 32, 900), (1024, 900, 48, 900), (1024, 30, 49, 100), (1025, 5, 8, 9000), (5, 1025, 8, 300), (1024, 2048, 33, 2500), (700, 2049, 6, 0),
                                               (2049, 2049, 4, 100), (30000, 35535, 2, 70000), (65534, 1, 1, 3), (1, 65534, 3, 150000)])
@pytest.mark.parametrize("window", [0, 30])
def test_remap_of_large_batches(old, B, width, slack, window, pkg):  # noqa: F811
    r = np.random.default_rng(old + B)
    held = r.integers(0, width + 1, old)
    NP = int(held.sum()) + slack
    at, ids = np.concatenate([[0], np.cumsum(held)]), r.permutation(NP)
    table = np.where(np.arange(width) < held[:, None], ids[np.minimum(at[:-1, None] + np.arange(width), NP - 1)], -1).astype(np.int32)
    table[1::3] = table[:-1:3][:len(table[1::3])]           # every third row holds what its neighbour does
    held[1::3] = held[:-1:3][:len(held[1::3])]
    refs = refs_of(table, NP)
    lens = np.maximum(held * 16 - r.integers(0, 16, old), 0)
    sources = r.integers(-1, old, B)
    new_lens = np.where(sources >= 0, lens[np.maximum(sources, 0)], 0) + r.integers(0, 20, B)
    check_remap(pkg, table, refs, sources, lens, new_lens, alias=window > 0, window=window or None)


def test_remap_of_more_rows_than_fit(pkg):  # noqa: F811
    t, c = dev(np.full((65535, 1), -1)), dev(np.zeros(8))
    with pytest.raises(pkg.AdaspecError):
        pkg.kv_remap(t, c, dev([0]), dev(np.zeros(65535)), dev([0]))


@pytest.mark.parametrize("NP", [16384, 16385, 1 << 20, 1 << 21])
@pytest.mark.parametrize("alias", [False, True])
def test_compact_of_large_pools(NP, alias, pkg):  # noqa: F811
    r = np.random.default_rng(NP)
    for share in (0.3, 0.9995):
        ids = r.permutation(NP)[:int(share * NP)]
        table = np.concatenate([ids, np.full(-len(ids) % 64, -1)]).reshape(64, -1).astype(np.int32)
        refs = refs_of(table, NP)
        check_compact(pkg, table, refs, alias=alias)
        check_compact(pkg, table, refs, max_moves=77, alias=alias)


@pytest.mark.parametrize("NP", [5000, 50000])
def test_compact_of_a_table_with_millions_of_entries(NP, pkg):  # noqa: F811
    """More entries than the workgroups of one launch take at a time; every page in many of them, ids outside the pool too."""
    r = np.random.default_rng(NP)
    table = r.integers(-3, NP + 3, (601, 8192)).astype(np.int32)
    refs = np.bincount(table[(table >= 0) & (table < NP)], minlength=NP).astype(np.int32)
    free = r.permutation(NP)[:NP // 3]
    table[np.isin(table, free)] = -1
    refs[free] = 0
    for alias in (False, True):
        check_compact(pkg, table, refs, alias=alias)


@pytest.mark.parametrize("NP", [3000, 40000])
def test_compact_replayed(NP, pkg):  # noqa: F811
    """In place, a few pages at a time, replayed between eager calls that use the same workspace."""
    import torch
    r = np.random.default_rng(NP)
    table, refs, _ = state(r, 30, 60, 16, NP - 1000)
    refs = np.concatenate([refs, np.zeros(max(0, NP - len(refs)), np.int32)])
    t, c = dev(table), dev(refs)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda").random_(0, 256)
    out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (len(refs), 40, 40, 2)]
    kw = dict(max_moves=40, out_table=t, out_refs=c, page_map=out[0], copy_src=out[1], copy_dst=out[2], status=out[3], workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pkg.kv_compact_pages(t, c, **kw)
    side.synchronize()
    t.copy_(dev(table)), c.copy_(dev(refs))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        pkg.kv_compact_pages(t, c, **kw)
    for _ in range(5):
        g.replay()
        pkg.kv_compact_pages(dev(table), dev(refs), max_moves=9, workspace=ws)
        torch.cuda.synchronize()
        table, refs, *rest = kv_compact_pages(table, refs, 40)
        assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(c.cpu().numpy(), refs)
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, rest))


def test_two_calls_at_once(pkg):  # noqa: F811
    """A remap of either form and a compaction on streams of their own, with workspaces of their own."""
    import torch
    jobs = []
    for old, B, width, slack in ((50, 60, 40, 900), (300, 300, 200, 5000), (0, 0, 0, 0)):
        ws, stream = torch.empty(8 << 20, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
        r = np.random.default_rng(old)
        table, refs, held = state(r, old or 100, width or 80, 16, slack or 9000)
        t, c = dev(table), dev(refs)
        if old:
            sources, lens = r.integers(-1, old, B), np.maximum(held * 16 - 3, 0)
            more = np.where(sources >= 0, lens[np.maximum(sources, 0)], 0) + r.integers(0, 40, B)
            ref = kv_remap(table, refs, sources, lens, more)
            ints = [dev(x) for x in (sources, lens, more)]
            call = lambda t=t, c=c, ints=ints, ws=ws: pkg.kv_remap(t, c, *ints, workspace=ws)             # noqa: E731
        else:
            ref = kv_compact_pages(table, refs, len(refs) // 2)
            call = lambda t=t, c=c, ws=ws: pkg.kv_compact_pages(t, c, workspace=ws)                       # noqa: E731
        jobs.append((call, ref, stream, []))
    torch.cuda.synchronize()
    for _ in range(8):
        for call, ref, stream, outs in jobs:
            with torch.cuda.stream(stream):
                outs.append(call())
    torch.cuda.synchronize()
    for _, ref, _, outs in jobs:
        for out in outs:
            assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(out, ref))
