"""Portable verification attention (csrc/attn_vector.hip), over a cache of the queries' type and over one in 8 bits: rows whose first tokens all
score NaN, and rows that see nothing of a split.

The cache of the queries' type holds the values that the one in 8 bits stands for (scales are powers of two: exact in bf16, fp16 and fp32), so
both have the same oracle in 64 bits.  Tolerance on the fp32 accumulator: 2e-5 for values of unit size, that of the other attention tests."""
import numpy as np
import pytest

from oracle import positions as P
from tests.ragged_rows import cache8, dev, host, ints, store, table, tree
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

TOL = 2e-5


def make(seed, ctx, spec, hq, hkv, d, dtype, is_tree=False, width=None):
    rng = np.random.default_rng(seed)
    bt, num = table(rng, ctx, width=width)
    (k8, ks), (v8, vs) = cache8(rng, num, hkv, d), cache8(rng, num, hkv, d)
    q = store(rng.normal(0, 1, (sum(spec) + len(spec), hq, d)), dtype)
    return dict(q=q, k8=k8.copy(), v8=v8.copy(), ks=ks, vs=vs, bt=bt, ctx=ctx, spec=spec, dtype=dtype, parents=tree(rng, spec) if is_tree else None)


def both(pkg, c):  # noqa: F811
    """(name, output in fp32) of the two calls; the table is as wide as it was made"""
    import torch
    kw = dict(max_spec_len=max(c["spec"]), parents=None if c["parents"] is None else dev(c["parents"]), out_dtype=0, path="vector")
    where = dev(c["bt"]), ints(*c["ctx"]), ints(*c["spec"])
    q = dev(c["q"], c["dtype"])
    k, v = (store(P.E4M3[x8] * s[..., None, None], c["dtype"]) for x8, s in ((c["k8"], c["ks"]), (c["v8"], c["vs"])))
    outs = [("wide", pkg.verify_attn(q, dev(k, c["dtype"]), dev(v, c["dtype"]), *where, **kw)),
            ("8 bits", pkg.verify_attn(q, dev(c["k8"], "e4m3"), dev(c["v8"], "e4m3"), *where, k_scales=dev(c["ks"]), v_scales=dev(c["vs"]), **kw))]
    torch.cuda.synchronize()
    return [(name, host(o).astype(np.float64)) for name, o in outs]


def check(pkg, c, nan):  # noqa: F811
    ref = P.verify_attn_scaled(c["q"], c["k8"], c["v8"], c["ks"], c["vs"], c["bt"], c["ctx"], c["spec"], dtype=c["dtype"], parents=c["parents"])
    assert np.isnan(ref).any() == nan
    for name, out in both(pkg, c):
        assert np.array_equal(np.isnan(out), np.isnan(ref)), name
        assert (np.abs(out - ref) <= TOL)[~np.isnan(ref)].all(), name


@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("d,dtype", [(96, "bf16"), (96, "f32"), (64, "f16"), (256, "bf16")])
def test_the_first_tokens_score_nan(d, dtype, is_tree, pkg):  # noqa: F811
    """All 64 tokens of a block, the first split whole, a split in the middle: the rows that see them are NaN."""
    c = make(3, [200, 700, 900, 40], [3, 2, 5, 1], 4, 2, d, dtype, is_tree)
    for i, t0, t1, head in ((0, 0, 64, 1), (1, 0, 256, 0), (2, 256, 512, 1)):
        for t in range(t0, t1):
            c["k8"][c["bt"][i, t // 16], head, t % 16, t % d] = 0x7f
    check(pkg, c, True)


@pytest.mark.parametrize("d,dtype", [(96, "bf16"), (96, "f32"), (64, "f16"), (256, "bf16")])
@pytest.mark.parametrize("shape", [([769], [5]), ([769, 257, 30], [4, 80, 0]), ([2305], [9])], ids=lambda s: f"L{max(s[0])}-k{max(s[1])}")
def test_rows_that_see_nothing_of_a_split(shape, d, dtype, pkg):  # noqa: F811
    """The last split holds drafts alone, under a table wide enough for many splits; few rows, joined by four wavefronts each."""
    check(pkg, make(5, *shape, 2, 2, d, dtype, width=160), False)


@pytest.mark.parametrize("d,dtype", [(96, "bf16"), (64, "f16")])
def test_nodes_that_see_nothing_of_a_split(d, dtype, pkg):  # noqa: F811
    check(pkg, make(6, [769, 1025], [5, 63], 2, 2, d, dtype, True, width=160), False)
