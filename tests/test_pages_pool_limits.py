"""How many pages a pool may have, on the host: no call of this file gets as far as a kernel."""
import ctypes as C

import pytest

import paper_2503_05096_amd as pkg
from tests.test_pages_abi import _compact, _pages, _remap

INT_MAX = (1 << 31) - 1


@pytest.mark.parametrize("pages", [(1 << 24) + 1, 1 << 30, INT_MAX - 1024, INT_MAX - 1023, INT_MAX - 1022, INT_MAX])
def test_pools_too_large(pages):
    """(from INT_MAX - 1022 on the number of chunks of 1024 pages used to overflow, and with it the workspace's size)"""
    d = _pages(num_pages=pages)
    assert pkg.lib().adaspec_kv_remap_workspace_bytes(C.byref(d)) == 0 and _remap(d) == -6
    assert pkg.lib().adaspec_kv_compact_pages_workspace_bytes(C.byref(d)) == 0 and _compact(d) == -6


@pytest.mark.parametrize("size,most,per_page", [("adaspec_kv_remap_workspace_bytes", 1 << 24, 8),
                                                ("adaspec_kv_compact_pages_workspace_bytes", 1 << 21, 0.25)])
def test_largest_pools(size, most, per_page):
    d = _pages(num_pages=most)
    assert getattr(pkg.lib(), size)(C.byref(d)) >= most * per_page
    call = _remap if "remap" in size else _compact
    assert call(d, nbytes=0) == -5                      # refused for its workspace, not for its size


@pytest.mark.gpu
@pytest.mark.parametrize("old", [1, 1100])              # (both forms)
def test_remap_of_the_largest_pool(old):
    """Free pages at its far end only, and fewer than wanted: handed out in ascending order."""
    import torch
    NP, width = 1 << 24, 6
    print(f"[case] remap pool={NP} old={old}", flush=True)
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")                         # noqa: E731
    refs = torch.ones(NP, dtype=torch.int32, device="cuda")
    free = torch.arange(NP - 1, NP - 600, -2, device="cuda").flip(0)
    refs[free] = 0
    table = torch.full((old, width), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 5                                     # one page of an old row that ends: free again
    new_lens = dev(*[16 * (k % 7) for k in range(200)])
    out, new_refs, src, dst, status = pkg.kv_remap(table, refs, torch.full_like(new_lens, -1), dev(*[0] * old), new_lens)
    free = torch.cat([dev(5), free.int()])
    wants = torch.arange(width, device="cuda") < (new_lens[:, None] // 16)
    expected = torch.full((200, width), -1, dtype=torch.int32, device="cuda")
    served = wants & (wants.reshape(-1).cumsum(0).view_as(wants) <= len(free))
    expected[served] = free[:int(served.sum())]
    assert torch.equal(out, expected) and status.tolist() == [0, int(wants.sum()) - len(free)]
    refs[5] = 0
    refs[expected[served].long()] = 1
    assert torch.equal(new_refs, refs) and (src == -1).all() and (dst == -1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("width", [400, 500])           # (in two launches, in four)
def test_remap_in_a_large_pool(width):
    import numpy as np

    from tests.test_gpu_kv_pages import check_remap, state
    r = np.random.default_rng(width)
    table, refs, held = state(r, 64, width, 16, slack=0)
    ids = np.sort(r.permutation(1 << 20)[:len(refs)])   # the same batch with its pages all over a larger pool
    table = np.where(table >= 0, ids[np.maximum(table, 0)], -1).astype(np.int32)
    pool = (r.random(1 << 20) < 0.9).astype(np.int32)
    pool[ids] = refs
    lens = np.minimum(r.integers(0, width * 16 + 1, 64), held * 16)
    sources = r.integers(-1, 64, 64)
    new_lens = np.where(sources >= 0, lens[np.maximum(sources, 0)], 0) + r.integers(0, 60, 64)
    print(f"[case] remap pool={len(pool)} width={width}", flush=True)
    check_remap(pkg, table, pool, sources, lens, new_lens, window=900, sinks=20)
