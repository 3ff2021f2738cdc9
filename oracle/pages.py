"""CPU oracle of the pages of the cache: who holds which after a step, compaction, and the copies of K/V.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain loops, in the order in which the rules are stated; integers and
bytes, so every result is exact."""
from __future__ import annotations

import numpy as np


def refs_of(table, num_pages):
    refs = np.zeros(num_pages, np.int32)
    for p in np.asarray(table).reshape(-1):
        if 0 <= p < num_pages:
            refs[p] += 1
    return refs


def kv_remap(block_table, page_refs, sources, lens, new_lens, *, window=0, sinks=0, page_size=16):
    """(out_table, out_refs, copy_src, copy_dst, status)"""
    old, width = block_table.shape
    NP, B, P = len(page_refs), len(sources), page_size
    refs = page_refs.astype(np.int64).copy()
    held = lambda p: 0 <= p < NP                                                               # noqa: E731
    cut = lambda n: min(max(int(n), 0), width * P)                                             # noqa: E731
    for row in block_table:
        for p in row:
            if held(p):
                refs[p] -= 1
    out = np.full((B, width), -1, np.int32)
    kept = [cut(lens[s]) if 0 <= s < old else 0 for s in sources]
    for i, s in enumerate(sources):
        for j in range(-(-kept[i] // P)):
            behind = window > 0 and j * P >= sinks and j * P + P - 1 <= kept[i] - window
            if not behind and held(block_table[s, j]):
                out[i, j] = block_table[s, j]
                refs[out[i, j]] += 1
    free = [p for p in range(NP) if refs[p] == 0]
    shared = refs.copy()
    wants = []                                      # (row, entry, shared page or -1)
    for i in range(B):
        n = kept[i]
        if n % P and new_lens[i] > n:
            p = out[i, n // P]
            if p >= 0 and shared[p] > 1:
                shared[p] -= 1
                wants.append((i, n // P, int(p)))
        wants += [(i, j, -1) for j in range(-(-n // P), -(-cut(new_lens[i]) // P))]
    copy_src, copy_dst = np.full(B, -1, np.int32), np.full(B, -1, np.int32)
    for (i, j, p), f in zip(wants, free):
        out[i, j] = f
        refs[f] += 1
        if p >= 0:
            refs[p] -= 1
            copy_src[i], copy_dst[i] = p, f
    status = np.array([max(0, len(free) - len(wants)), max(0, len(wants) - len(free))], np.int32)
    return out, refs.astype(np.int32), copy_src, copy_dst, status


def kv_compact_pages(block_table, page_refs, max_moves):
    """(out_table, out_refs, page_map, copy_src, copy_dst, status)"""
    NP = len(page_refs)
    used = [p for p in range(NP) if page_refs[p] > 0]
    N = len(used)
    movers, holes = [p for p in used if p >= N], [p for p in range(N) if page_refs[p] <= 0]
    assert len(movers) == len(holes)
    done = list(zip(movers, holes))[:max_moves]
    to = dict(done)
    refs, page_map = page_refs.copy(), np.full(NP, -1, np.int32)
    for p in used:
        page_map[p] = to.get(p, p)
    for p, f in done:
        refs[f], refs[p] = page_refs[p], 0
    table = np.vectorize(lambda p: to.get(int(p), int(p)), otypes=[np.int32])(block_table) if block_table.size else block_table.copy()
    pairs = np.full((2, max_moves), -1, np.int32)
    for m, (p, f) in enumerate(done):
        pairs[0, m], pairs[1, m] = p, f
    return table, refs, page_map, pairs[0], pairs[1], np.array([N, len(movers)], np.int32)


def kv_copy_pages(pages, copy_src, copy_dst):
    """A copy of `pages` [..., num_pages, Hkv, P, d] with the pairs' pages copied."""
    out = pages.copy()
    NP = pages.shape[-4]
    for s, t in zip(copy_src, copy_dst):
        if 0 <= s < NP and 0 <= t < NP:
            out[..., t, :, :, :] = pages[..., s, :, :, :]
    return out
