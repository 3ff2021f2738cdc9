"""What adaspec_kv_remap, adaspec_kv_compact_pages and adaspec_kv_copy_pages refuse, on the host: no call of this file gets as
far as a kernel."""
import ctypes as C

import pytest

import paper_2503_05096_amd as pkg
from paper_2503_05096_amd.binding import BF16, CopyDims, PagesDims

# stand-ins for device arrays, far apart and never dereferenced
PTRS = [0x100000000 * (k + 1) for k in range(11)]


def _pages(**kw):
    base = dict(batch=3, old_batch=2, max_pages_per_req=8, num_pages=64, page_size=16, window=0, sinks=0, max_moves=32)
    base.update(kw)
    return PagesDims(**base)


def _remap(d, ptrs=None, ws=PTRS[10], nbytes=1 << 40):
    return pkg.lib().adaspec_kv_remap(*(ptrs or PTRS[:10]), C.byref(d), ws, nbytes, None)


def _compact(d, ptrs=None, ws=PTRS[10], nbytes=1 << 40):
    return pkg.lib().adaspec_kv_compact_pages(*(ptrs or PTRS[:8]), C.byref(d), ws, nbytes, None)


SHARED = [(dict(old_batch=-1), -2), (dict(max_pages_per_req=0), -2), (dict(num_pages=0), -2), (dict(num_pages=-5), -2),
          (dict(page_size=0), -2), (dict(max_pages_per_req=1 << 27, page_size=16), -6)]


@pytest.mark.parametrize("kw,code", SHARED + [(dict(batch=-1), -2), (dict(window=-1), -2), (dict(sinks=-1), -2),
                                              (dict(batch=65000, old_batch=600), -6), (dict(batch=60000, max_pages_per_req=1 << 15), -6)])
def test_remap_rejects_bad_dims(kw, code):
    d = _pages(**kw)
    assert _remap(d) == code and pkg.lib().adaspec_kv_remap_workspace_bytes(C.byref(d)) == 0


@pytest.mark.parametrize("kw,code", SHARED + [(dict(max_moves=0), -2), (dict(max_moves=65), -2), (dict(num_pages=(1 << 21) + 1), -6)])
def test_compact_rejects_bad_dims(kw, code):
    d = _pages(**kw)
    assert _compact(d) == code and pkg.lib().adaspec_kv_compact_pages_workspace_bytes(C.byref(d)) == 0


def test_pointers_workspaces_and_overlaps():
    L, d = pkg.lib(), _pages()
    assert L.adaspec_kv_remap(*PTRS[:10], None, PTRS[10], 1 << 40, None) == -1
    assert L.adaspec_kv_compact_pages(*PTRS[:8], None, PTRS[10], 1 << 40, None) == -1
    for call, n, size in ((_remap, 10, L.adaspec_kv_remap_workspace_bytes), (_compact, 8, L.adaspec_kv_compact_pages_workspace_bytes)):
        for k in range(n):
            p = PTRS[:n]
            p[k] = None
            assert call(d, p) == -1, k
        assert call(d, ws=None) == -1 and call(d, ws=PTRS[10] + 128) == -4
        need = size(C.byref(d))
        assert need > 0 and need % 256 == 0 and call(d, nbytes=need - 1) == -5
    table, refs = 2 * 8 * 4, 64 * 4
    # (arguments: block_table, page_refs, sources, lens, new_lens, out_table, out_refs, ...)
    for at, to, by in ((5, 0, 0), (5, 0, table - 4), (6, 1, 4), (6, 1, refs - 4)):
        p = PTRS[:10]
        p[at] = p[to] + by
        assert _remap(d, p) == -2, (at, by)
    p = PTRS[:10]
    p[5] = p[0] - 3 * 8 * 4 + 4                     # the end of the new table over the start of the old one
    assert _remap(d, p) == -2
    for at, to, by in ((2, 0, 4), (2, 0, table - 4), (3, 1, 4)):
        p = PTRS[:8]
        p[at] = p[to] + by
        assert _compact(d, p) == -2, (at, by)


def test_outputs_over_anything_else():
    """Every output over every other array, at its beginning and at its last entry; what may be the same array may not be so
    shifted."""
    d = _pages()
    need = [pkg.lib().adaspec_kv_remap_workspace_bytes(C.byref(d)), pkg.lib().adaspec_kv_compact_pages_workspace_bytes(C.byref(d))]
    # entries of every argument, and which of them are outputs
    for call, entries, outs, same, ws in ((_remap, [16, 64, 3, 2, 3, 24, 64, 3, 3, 2], range(5, 10), [(6, 1)], need[0]),
                                          (_compact, [16, 64, 16, 64, 64, 32, 32, 2], range(2, 8), [(2, 0), (3, 1)], need[1])):
        for o in outs:
            for k in range(len(entries)):
                for by in (0, 4 * (entries[k] - 1)):
                    if k == o or (by == 0 and (o, k) in same):
                        continue
                    p = PTRS[:len(entries)]
                    p[o] = p[k] + by
                    assert call(d, p) == -2, (call.__name__, o, k, by)
            p = PTRS[:len(entries)]
            p[o] = PTRS[10] + ws - 4
            assert call(d, p) == -2, o
        for k in range(len(entries)):
            p = PTRS[:len(entries)]
            p[k] = PTRS[10]
            assert call(d, p) == -2, k


@pytest.mark.parametrize("kw,n,code", [
    (dict(layers=-1), 4, -2), (dict(num_pages=0), 4, -2), (dict(n_kv_heads=0), 4, -2), (dict(page_size=-1), 4, -2), (dict(head_dim=0), 4, -2),
    (dict(), -1, -2), (dict(dtype=5), 4, -3), (dict(head_dim=12), 4, -6), (dict(head_dim=6, dtype=0), 4, -6),
    (dict(n_kv_heads=1 << 16, page_size=1 << 10), 4, -6),
])
def test_copy_rejects_bad_dims(kw, n, code):
    base = dict(layers=2, num_pages=64, n_kv_heads=8, page_size=16, head_dim=128, dtype=BF16)
    base.update(kw)
    assert pkg.lib().adaspec_kv_copy_pages(*PTRS[:4], n, C.byref(CopyDims(**base)), None) == code


def test_copy_pointers_and_calls_that_copy_nothing():
    L, d = pkg.lib(), CopyDims(2, 64, 8, 16, 128, BF16)
    assert L.adaspec_kv_copy_pages(*PTRS[:4], 4, None, None) == -1
    for k in range(4):
        p = PTRS[:4]
        p[k] = None
        assert L.adaspec_kv_copy_pages(*p, 4, C.byref(d), None) == -1
    for k in range(2):
        p = PTRS[:4]
        p[k] += 8
        assert L.adaspec_kv_copy_pages(*p, 4, C.byref(d), None) == -4
    assert L.adaspec_kv_copy_pages(None, None, None, None, 0, C.byref(d), None) == 0
    d.layers = 0
    assert L.adaspec_kv_copy_pages(None, None, None, None, 4, C.byref(d), None) == 0


def test_python_refusals():
    import torch
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError, match="window"):
        pkg.kv_remap(t, t[0], t[0, :2], t[0, :2], t[0, :2], sinks=4)
    with pytest.raises(ValueError, match="window"):
        pkg.kv_remap(t, t[0], t[0, :2], t[0, :2], t[0, :2], window=0)
    with pytest.raises(AssertionError):             # not on a GPU
        pkg.kv_remap(t, t[0], t[0, :2], t[0, :2], t[0, :2])
    with pytest.raises(AssertionError):
        pkg.kv_compact_pages(t, t[0])
    with pytest.raises(AssertionError):
        pkg.kv_copy_pages(torch.zeros(3, 1, 16, 8), torch.zeros(3, 1, 16, 8), t[0], t[0])
