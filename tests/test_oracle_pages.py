"""The oracle of the cache's pages (oracle/pages.py), by hand and by what has to hold after every call."""
import numpy as np
import pytest

from oracle.pages import kv_compact_pages, kv_copy_pages, kv_remap, refs_of


def ints(*v):
    return np.array(v, np.int32)


def test_by_hand():
    # two requests of 20 and 32 tokens, a third entry of the first reserved for drafts that were rejected
    table = ints([5, 2, 7, -1], [2, 6, -1, -1])     # page 2 is shared
    refs = refs_of(table, 8)
    assert refs.tolist() == [0, 0, 2, 0, 0, 1, 1, 1]
    # the first forks into three samples, the second ends, a new one of 17 tokens starts
    out, r, src, dst, status = kv_remap(table, refs, ints(0, 0, -1, 0), ints(20, 32), ints(21, 33, 17, 20))
    # free then: 0 1 3 4 6 7; page 2 (tokens 16..) has 3 holders: rows 0 and 1 want their own, row 3 writes nothing
    assert src.tolist() == [2, 2, -1, -1] and dst.tolist() == [0, 1, -1, -1]
    assert out.tolist() == [[5, 0, -1, -1], [5, 1, 3, -1], [4, 6, -1, -1], [5, 2, -1, -1]]
    assert r.tolist() == [1, 1, 1, 1, 1, 3, 1, 0] and status.tolist() == [1, 0]
    # a window of 8 with 4 sinks at 40 tokens: entry 1 (tokens 16..31) is behind it (32 is not: 33..40 is seen next)
    table = ints([3, 4, 5])
    out, r, *_ = kv_remap(table, refs_of(table, 6), ints(0), ints(40), ints(41), window=8, sinks=4)
    assert out.tolist() == [[3, -1, 5]] and r.tolist() == [0, 0, 0, 1, 0, 1]
    out, *_ = kv_remap(table, refs_of(table, 6), ints(0), ints(38), ints(38), window=8, sinks=4)     # tokens 31.. are seen next
    assert out.tolist() == [[3, 4, 5]]
    out, *_ = kv_remap(table, refs_of(table, 6), ints(0), ints(40), ints(40), window=8, sinks=0)
    assert out.tolist() == [[-1, -1, 5]]


def test_wants_that_cannot_be_served_are_served_by_the_next_call():
    table = ints([0, 1, -1, -1])
    out, r, src, dst, status = kv_remap(table, refs_of(table, 3), ints(0, 0), ints(20), ints(50, 21))
    assert status.tolist() == [0, 2]                # a copy, two fresh pages; the last keeps page 1
    assert out.tolist() == [[0, 2, -1, -1], [0, 1, -1, -1]] and src.tolist() == [1, -1] and dst.tolist() == [2, -1]
    more = np.concatenate([r, ints(0, 0)])
    out, r, src, dst, status = kv_remap(out, more, ints(0, 1), ints(20, 20), ints(50, 21))
    assert out.tolist() == [[0, 2, 3, 4], [0, 1, -1, -1]] and status.tolist() == [0, 0] and (src < 0).all()


@pytest.mark.parametrize("seed", range(20))
def test_what_holds_after_a_remap(seed):
    r = np.random.default_rng(seed)
    old, B, width, P = int(r.integers(1, 6)), int(r.integers(1, 9)), 7, 4
    held = r.integers(0, width + 1, old)
    NP = int(held.sum()) + int(r.integers(1, 30))
    ids = r.permutation(NP)
    table = np.full((old, width), -1, np.int32)
    for i in range(old):
        table[i, :held[i]] = ids[held[:i].sum():held[:i + 1].sum()]
    if old > 1:
        both = min(held[0], held[1])
        table[1, :both // 2] = table[0, :both // 2]
    refs = refs_of(table, NP)
    outside = r.integers(0, NP)
    refs[outside] += 1                              # somebody else holds a page
    lens = np.minimum(r.integers(0, width * P + 1, old), held * P)
    sources = r.integers(-1, old, B)
    kept = np.where(sources >= 0, lens[np.maximum(sources, 0)], 0)
    new_lens = np.minimum(kept + r.integers(0, 10, B), width * P)
    out, after, src, dst, status = kv_remap(table, refs, sources, lens, new_lens, page_size=P)
    mine = refs_of(out, NP)
    mine[outside] += 1
    assert np.array_equal(after, mine)              # the counts are the holders
    assert status[0] == (after == 0).sum()
    if status[1] == 0:
        for i in range(B):
            assert (out[i, :-(-new_lens[i] // P)] >= 0).all()
            for j in range(kept[i] // P, -(-new_lens[i] // P)):
                if new_lens[i] > kept[i]:
                    assert after[out[i, j]] == 1    # whatever is written next has one holder
    for s, t in zip(src, dst):
        assert (s < 0) == (t < 0)
        assert t < 0 or (t not in src and (dst == t).sum() == 1 and after[s] >= 1)


def test_compaction_by_hand():
    table, refs = ints([1, 7], [7, 4], [-1, 9]), ints(0, 1, 0, 0, 1, 0, 0, 2, 0, 1)
    out, r, m, src, dst, status = kv_compact_pages(table, refs, 5)
    assert status.tolist() == [4, 3] and src.tolist() == [4, 7, 9, -1, -1] and dst.tolist() == [0, 2, 3, -1, -1]
    assert out.tolist() == [[1, 2], [2, 0], [-1, 3]] and r.tolist() == [1, 1, 2, 1, 0, 0, 0, 0, 0, 0]
    assert m.tolist() == [-1, 1, -1, -1, 0, -1, -1, 2, -1, 3]
    out, r, m, src, dst, status = kv_compact_pages(table, refs, 1)
    assert status.tolist() == [4, 3] and (src.tolist(), dst.tolist()) == ([4], [0]) and out.tolist() == [[1, 7], [7, 0], [-1, 9]]
    k = np.arange(10.0).reshape(10, 1, 1, 1)
    assert kv_copy_pages(k, ints(4, 7, -1), ints(0, 2, 3)).reshape(-1).tolist() == [4, 1, 7, 3, 4, 5, 6, 7, 8, 9]
