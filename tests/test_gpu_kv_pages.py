"""The pages of the cache on the GPU (csrc/kv_pages.hip) against the oracle: integers and bytes, so everything is equal."""
import numpy as np
import pytest

from oracle.pages import kv_compact_pages, kv_copy_pages, kv_remap, refs_of
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def state(r, old, width, P, slack=20, share=0.5, extra=0, held=None):
    """(table, refs): rows of any length, some beginning like another one, pages held from outside"""
    held = r.integers(0, width + 1, old) if held is None else held
    NP = int(held.sum()) + slack
    ids = r.permutation(NP)
    at = np.concatenate([[0], np.cumsum(held)])
    table = np.full((old, width), -1, np.int32)
    for i in range(old):
        table[i, :held[i]] = ids[at[i]:at[i + 1]]
        if i and r.random() < share:
            j = int(r.integers(0, i))
            both = min(held[i], held[j])
            n = int(r.integers(0, both + 1))
            table[i, :n] = table[j, :n]
        if held[i] > 3 and r.random() < 0.3:
            table[i, 1:3] = -1                      # given back earlier
    refs = refs_of(table, NP)
    for _ in range(extra):
        refs[r.integers(0, NP)] += 1
    return table, refs, held


def check_remap(pkg, table, refs, sources, lens, new_lens, alias=False, **kw):  # noqa: F811
    import torch
    ref = kv_remap(table, refs, sources, lens, new_lens, window=kw.get("window") or 0, sinks=kw.get("sinks", 0), page_size=kw.get("page_size", 16))
    t, c = dev(table), dev(refs)
    got = pkg.kv_remap(t, c, dev(sources), dev(lens), dev(new_lens), out_refs=c if alias else None, **kw)
    torch.cuda.synchronize()
    for name, a, b in zip(("table", "refs", "copy_src", "copy_dst", "status"), got, ref):
        assert np.array_equal(a.cpu().numpy(), b), name
    assert np.array_equal(t.cpu().numpy(), table)   # the old table stays
    assert alias or np.array_equal(c.cpu().numpy(), refs)
    return got


@pytest.mark.parametrize("seed", range(12))
def test_remap(seed, pkg):  # noqa: F811
    r = np.random.default_rng(seed)
    for old, B, width, P, slack in ((1, 1, 1, 16, 1), (3, 5, 9, 16, 40), (40, 70, 33, 4, 300), (300, 300, 5, 16, 900), (17, 600, 12, 1, 2000),
                                    (2, 3, 5000, 2, 50), (60, 61, 80, 16, 4500), (5, 4, 20, 16, 0)):
        table, refs, held = state(r, old, width, P, slack, extra=seed % 3)
        lens = np.minimum(r.integers(0, width * P + 1, old), held * P)
        sources = r.integers(-2, old + 1, B)        # (also rows that there are not)
        kept = np.where((sources >= 0) & (sources < old), lens[np.clip(sources, 0, old - 1)], 0)
        new_lens = kept + r.integers(-3, 3 * P + 2, B)
        kw = dict(page_size=P)
        if seed % 2:
            kw.update(window=int(r.integers(1, width * P + 1)), sinks=int(r.integers(0, 3 * P)))
        print(f"[case] remap seed={seed} {old}->{B} x{width} P={P} pages={len(refs)} {kw}", flush=True)
        check_remap(pkg, table, refs, sources, lens, new_lens, alias=seed % 4 == 0, **kw)


@pytest.mark.parametrize("NP", [1, 2, 255, 256, 4095, 4096, 4097, 12289])
def test_remap_pool_sizes(NP, pkg):  # noqa: F811
    r = np.random.default_rng(NP)
    refs = (r.random(NP) < 0.6).astype(np.int32)    # all held from outside
    table = np.full((1, 40), -1, np.int32)
    for wants in (0, 1, 17, 40):
        check_remap(pkg, table, refs, np.array([-1]), np.array([0]), np.array([wants * 16]))
    check_remap(pkg, table, refs, np.full(100, -1), np.array([0]), np.full(100, 640))


def test_remap_without_rows(pkg):  # noqa: F811
    r = np.random.default_rng(3)
    table, refs, held = state(r, 6, 8, 16)
    check_remap(pkg, table, refs, np.zeros(0), held * 16, np.zeros(0))              # everybody has ended
    empty = np.zeros((0, 8), np.int32)
    check_remap(pkg, empty, refs, np.array([-1, 4]), np.zeros(0), np.array([20, 128]))
    check_remap(pkg, empty, refs, np.zeros(0), np.zeros(0), np.zeros(0))


def test_remap_one_page_shared_by_many(pkg):  # noqa: F811
    """Forks of one row, each about to write; of two rows that share a page and both write; with a holder outside."""
    for extra in (0, 1):
        table = np.array([[3, 1, -1, -1], [3, 1, 2, -1]], np.int32)
        refs = refs_of(table, 900)
        refs[1] += extra
        sources = np.array([0, 1] * 300)
        lens = np.array([20, 24])
        for grow in (0, 1, 30):
            new_lens = np.where(np.arange(600) % 5 == 0, lens[sources], lens[sources] + grow)
            check_remap(pkg, table, refs, sources, lens, new_lens)


def test_remap_entries_and_lengths_that_make_no_sense(pkg):  # noqa: F811
    """Ids outside the pool hold nothing, lengths are cut to the row."""
    table = np.array([[70, 1, -9, 2], [1 << 30, -(1 << 31), 3, 64]], np.int32)
    refs = refs_of(table, 64)
    big = (1 << 31) - 1
    check_remap(pkg, table, refs, np.array([0, 1, 1, big, -(1 << 31)]), np.array([big, -5]), np.array([big, -(1 << 31), 1, 40, 20]))
    check_remap(pkg, table, refs, np.array([0, 1]), np.array([60, big]), np.array([64, big]), window=big, sinks=big)
    check_remap(pkg, table, refs, np.array([0, 1]), np.array([60, big]), np.array([64, big]), window=1, sinks=0)


def test_remap_replayed(pkg):  # noqa: F811
    """A captured pair of calls, there and back between two tables, counts in place, replayed between eager calls that use the
    same workspace."""
    import torch
    r = np.random.default_rng(8)
    table, refs, held = state(r, 12, 20, 16, 400, share=0)
    lens = np.where(held > 0, held * 16 - 5, 0)
    sources = r.integers(0, 12, 12)
    a, b, c = dev(table), torch.empty_like(dev(table)), dev(refs)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda").random_(0, 256)
    ints = [dev(x) for x in (sources, lens, lens[sources] + 3)]
    ident, ones = dev(np.arange(12)), [torch.empty(12, dtype=torch.int32, device="cuda") for _ in range(2)]
    status = torch.empty(2, dtype=torch.int32, device="cuda")

    def pair():
        pkg.kv_remap(a, c, ints[0], ints[1], ints[2], out_table=b, out_refs=c, copy_src=ones[0], copy_dst=ones[1], status=status, workspace=ws)
        pkg.kv_remap(b, c, ident, ints[2], ints[2], out_table=a, out_refs=c, copy_src=ones[0], copy_dst=ones[1], status=status, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pair()
    side.synchronize()
    a.copy_(dev(table)), c.copy_(dev(refs))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        pair()
    ht, hr = table, refs
    for _ in range(4):
        g.replay()
        check_remap(pkg, table, refs, sources, lens, lens[sources] + 9, workspace=ws)
        torch.cuda.synchronize()
        t, q, *_ = kv_remap(ht, hr, sources, lens, lens[sources] + 3)
        ht, hr, *_ = kv_remap(t, q, np.arange(12), lens[sources] + 3, lens[sources] + 3)
        assert np.array_equal(a.cpu().numpy(), ht) and np.array_equal(c.cpu().numpy(), hr)


def check_compact(pkg, table, refs, max_moves=None, alias=False):  # noqa: F811
    import torch
    most = max(1, len(refs) // 2) if max_moves is None else max_moves
    ref = kv_compact_pages(table, refs, most)
    t, c = dev(table), dev(refs)
    got = pkg.kv_compact_pages(t, c, max_moves=max_moves, **(dict(out_table=t, out_refs=c) if alias else {}))
    torch.cuda.synchronize()
    for name, a, b in zip(("table", "refs", "map", "copy_src", "copy_dst", "status"), got, ref):
        assert np.array_equal(a.cpu().numpy(), b), name
    return ref


@pytest.mark.parametrize("NP", [1, 2, 3, 64, 255, 257, 4095, 4096, 4097, 8192, 20001])
@pytest.mark.parametrize("alias", [False, True])
def test_compact(NP, alias, pkg):  # noqa: F811
    r = np.random.default_rng(NP)
    for share in (0.0, 0.02, 0.5, 0.97, 1.0):
        ids = r.permutation(NP)[:int(share * NP)]
        width = max(1, len(ids) // 3)
        table = np.full((4, width), -1, np.int32)
        table.reshape(-1)[r.permutation(4 * width)[:min(len(ids), 4 * width)]] = ids[:4 * width]
        refs = refs_of(table, NP)
        refs[ids[::7]] += 2                         # held from outside as well
        check_compact(pkg, table, refs, alias=alias)
        check_compact(pkg, table, refs, max_moves=min(NP, 1 + int(share * 10)), alias=alias)
        check_compact(pkg, table, refs, max_moves=NP, alias=alias)
    check_compact(pkg, np.zeros((0, 5), np.int32), refs, alias=alias)


def test_compact_step_by_step(pkg):  # noqa: F811
    r = np.random.default_rng(4)
    table, refs, _ = state(r, 30, 50, 16, 3000)
    for k in range(200):
        table, refs, page_map, src, dst, status = check_compact(pkg, table, refs, max_moves=37)
        if status[1] <= 37:
            break
    assert (refs[:status[0]] > 0).all() and (refs[status[0]:] == 0).all() and k > 3


@pytest.mark.parametrize("dtype,layers,hkv,P,d", [("bf16", None, 8, 16, 128), ("f16", 1, 2, 16, 64), ("f32", 3, 3, 16, 20), ("bf16", 5, 1, 1, 8),
                                                  ("f32", 2, 7, 5, 4), ("f16", 33, 2, 16, 96), ("bf16", None, 32, 16, 256)])
def test_copy_pages(dtype, layers, hkv, P, d, pkg):  # noqa: F811
    import torch
    r = np.random.default_rng(d)
    NP = 61
    shape = (() if layers is None else (layers,)) + (NP, hkv, P, d)
    raw = [r.integers(0, 256, shape + ({"f32": 4}.get(dtype, 2),), dtype=np.uint8) for _ in range(2)]       # any bytes, NaN among them
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    ids = r.permutation(NP)
    for n in (0, 1, 2, 30):
        src, dst = ids[:n].copy(), ids[30:30 + n].copy()
        if n == 30:                                 # pairs that are left out, one source several times, a page onto itself
            src[3], dst[4], src[5], dst[6], src[9] = -1, -1, NP, NP + 5, src[8]
            src[10] = dst[10]
        k, v = (torch.from_numpy(x.copy()).cuda().view(kind).reshape(shape) for x in raw)
        pkg.kv_copy_pages(k, v, dev(src), dev(dst))
        torch.cuda.synchronize()
        for got, x in zip((k, v), raw):
            want = kv_copy_pages(x.reshape(shape[:-1] + (-1,)), src, dst)
            assert np.array_equal(got.view(torch.uint8).cpu().numpy().reshape(want.shape), want), n


def test_copy_in_a_pool_beyond_32_bits(pkg):  # noqa: F811
    import torch
    NP = 140000                                     # 4.6 GB of K
    k, v = (torch.zeros((NP, 8, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for p in (NP - 1, 70000, 3):
        k[p], v[p] = p % 251, -(p % 241)
    src, dst = [NP - 1, 70000, 3], [0, NP - 2, 131073]
    pkg.kv_copy_pages(k, v, dev(src), dev(dst))
    torch.cuda.synchronize()
    for s, t in zip(src, dst):
        assert bool((k[t] == s % 251).all()) and bool((v[t] == -(s % 241)).all())
    assert int((k != 0).any(dim=3).any(dim=2).any(dim=1).sum()) == 6


def test_device_refusals(pkg):  # noqa: F811
    import torch
    t, c = dev(np.full((2, 4), -1)), dev(np.zeros(30))
    two = dev([0, 1])
    with pytest.raises(pkg.AdaspecError):
        pkg.kv_remap(t, c, two, two, two, out_table=t)
    with pytest.raises(pkg.AdaspecError):
        pkg.kv_remap(t, c, two, two, two, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    for bad in (dict(block_table=t.long()), dict(sources=two[:1]), dict(lens=dev([0, 1, 2])), dict(page_refs=c.view(2, 15)),
                dict(block_table=t.t()), dict(new_lens=two.cpu())):
        args = dict(block_table=t, page_refs=c, sources=two, lens=two, new_lens=two)
        args.update(bad)
        with pytest.raises((AssertionError, ValueError)):
            pkg.kv_remap(*args.values())
    with pytest.raises(AssertionError):
        pkg.kv_remap(t, c, two, two, two, out_table=torch.empty_like(t[:1]))
    with pytest.raises(pkg.AdaspecError):
        pkg.kv_compact_pages(t, c, max_moves=31)
    k = torch.zeros(4, 2, 16, 12, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(pkg.AdaspecError):
        pkg.kv_copy_pages(k, k.clone(), two, two)
    k = torch.zeros(4, 2, 16, 64, device="cuda")
    for args in ((k, k[:2], two, two), (k, k.half(), two, two), (k, k, two, dev([0])), (k, k, two.long(), two), (k[0], k[0], two, two),
                 (k.transpose(1, 2), k.transpose(1, 2), two, two)):
        with pytest.raises(AssertionError):
            pkg.kv_copy_pages(*args)
