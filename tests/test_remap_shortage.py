"""A remap whose wants are left over, and what may be written before the next one: followed token by token."""
import numpy as np
import pytest

from oracle.pages import kv_remap, refs_of

P = 4


class Pool:
    """What every slot of the pool holds, and what every row's tokens are."""

    def __init__(self, table, lens, num_pages):
        self.slots = np.full((num_pages, P), -1, np.int64)
        self.new = 0
        self.rows = []
        for row, n in zip(table, lens):
            for t in range(n):
                if self.slots[row[t // P], t % P] < 0:
                    self.write(row, t, t + 1)
            self.rows.append([self.slots[row[t // P], t % P] for t in range(n)])

    def write(self, row, begin, end):
        for t in range(begin, end):
            self.slots[row[t // P], t % P] = self.new
            self.new += 1
        return [self.slots[row[t // P], t % P] for t in range(begin, end)]

    def copy(self, src, dst):
        done = self.slots.copy()
        for s, t in zip(src, dst):
            if s >= 0:
                done[t] = self.slots[s]
        self.slots = done

    def check(self, table, rows):
        for i, tokens in enumerate(rows):
            assert [self.slots[table[i, t // P], t % P] for t in range(len(tokens))] == tokens, i


def may_be_written(table, refs, i, n, new):
    """The header's rule."""
    there = all(table[i, j] >= 0 for j in range(-(-new // P)))
    return there and (n % P == 0 or new <= n or refs[table[i, n // P]] == 1)


def steps(remap, table, refs, outside, lens, sources, grow):
    """A remap with pages held from outside, writes of the rows that may be written, a remap after those pages have come free"""
    pool = Pool(table, lens, len(refs))
    n = [lens[s] for s in sources]
    new = [a + g for a, g in zip(n, grow)]
    table, refs, src, dst, status = remap(table, refs, np.array(sources, np.int32), np.array(lens, np.int32), np.array(new, np.int32))
    short, rows = int(status[1]), [pool.rows[s][:a] for s, a in zip(sources, n)]
    pool.copy(src, dst)
    written = [may_be_written(table, refs, i, n[i], new[i]) for i in range(len(n))]
    for i, w in enumerate(written):
        if w:
            rows[i] = rows[i] + pool.write(table[i], n[i], new[i])
    pool.check(table, rows)
    refs = refs.copy()
    refs[outside] = 0
    lens2 = [len(r) for r in rows]
    table, refs, src, dst, status = remap(table, refs, np.arange(len(n), dtype=np.int32), np.array(lens2, np.int32), np.array(new, np.int32))
    assert status[1] == 0 and all(may_be_written(table, refs, i, lens2[i], new[i]) for i in range(len(n)))
    pool.copy(src, dst)
    for i in range(len(n)):
        rows[i] = rows[i] + pool.write(table[i], lens2[i], new[i])
    pool.check(table, rows)
    return short, written


def by_oracle(*args):
    return kv_remap(*args, page_size=P)


def batch(seed):
    """Two requests that share a page which is not full, at different lengths; others; pages held from outside"""
    r = np.random.default_rng(seed)
    width, num_pages = 8, 60
    table = np.full((3, width), -1, np.int32)
    table[0, :3], table[1, :3], table[2, :2] = (7, 3, 11), (7, 3, 11), (5, 20)
    lens = [int(8 + r.integers(1, 4)), int(8 + r.integers(1, 4)), int(r.integers(1, 8))]
    refs = refs_of(table, num_pages)
    free = r.permutation(np.nonzero(refs == 0)[0])
    outside = free[int(r.integers(0, 6)):]
    refs[outside] = 1
    sources = [0, 1] + [int(s) for s in r.integers(0, 3, int(r.integers(0, 4)))]
    r.shuffle(sources)
    return table, refs, outside, lens, sources, [int(g) for g in r.integers(0, 9, len(sources))]


def test_the_row_that_keeps_a_shared_page():
    """Rows of 10 and 9 tokens share page 11, the first gets no copy: the second may keep the page, but not write to it yet."""
    table = np.array([[7, 3, 11], [7, 3, 11]], np.int32)
    refs = refs_of(table, 13)
    outside = np.array([p for p in range(13) if refs[p] == 0])
    refs[outside] = 1
    out, out_refs, src, dst, status = by_oracle(table, refs, np.array([0, 1]), np.array([10, 9]), np.array([11, 10]))
    assert status.tolist() == [0, 1] and np.array_equal(out, table) and (src == -1).all()
    assert not may_be_written(out, out_refs, 0, 10, 11) and not may_be_written(out, out_refs, 1, 9, 10)
    short, written = steps(by_oracle, table, refs, outside, [10, 9], [0, 1], [1, 1])
    assert short == 1 and written == [False, False]


@pytest.mark.parametrize("seed", range(40))
def test_tokens_survive(seed):
    steps(by_oracle, *batch(seed))


def test_batches_are_short_of_pages():
    assert sum(steps(by_oracle, *batch(seed))[0] > 0 for seed in range(40)) >= 10


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(10))
def test_tokens_survive_on_the_gpu(seed):
    import torch

    import paper_2503_05096_amd as pkg

    def remap(*args):
        out = pkg.kv_remap(*(torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda() for a in args), page_size=P)
        return [t.cpu().numpy() for t in out]
    print(f"[case] shortage seed={seed}", flush=True)
    steps(remap, *batch(seed))
