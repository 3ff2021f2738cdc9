"""Attention over the cache in 8 bits on the matrix cores: the softmax weights cost the output nothing that fp32 shows.

Tolerance on the fp32 accumulator: 2e-5 for values of unit size, that of the other attention tests, where weights are fp32.  The weights
are two f16, the second what the first leaves: off by half a step of 11 bits, 2^-11, of at most 2^-11 of them, 2^-22, and a mean of values by up to
that times the mean of their magnitudes.  (One f16 alone would be off by up to 2^-11 of each weight.)"""
import numpy as np
import pytest

from tests.ragged_rows import HALF_STEP, LEAST, host, store, widen
from tests.test_gpu_attn_scaled import TOL, call, make, oracle
from tests.test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0 ** -22

SHAPES = [
    # ctx_lens, spec_lens, Hq, Hkv: one to four row tiles, two row groups
    ([1, 2, 16, 17, 31, 33, 64, 65, 63, 32], [0, 1, 0, 2, 1, 3, 0, 4, 0, 0], 2, 2),
    ([140, 257, 300, 19, 512, 1030], [3, 0, 5, 1, 7, 2], 8, 2),
    ([90, 700, 33], [10, 11, 0], 8, 2),
    ([400, 5, 90], [7, 3, 0], 14, 2),
    ([90, 700, 33], [10, 12, 0], 16, 2),
]


def check(pkg, c):  # noqa: F811
    ref, size = oracle(c)
    tol = TOL + WEIGHTS * size
    print(f"[case] attn8 {c['dtype']} {c['q'].shape} Hkv={c['k8'].shape[1]} B={len(c['ctx'])} tree={c['parents'] is not None}", flush=True)
    off = np.abs(host(call(pkg, c, out_dtype=0)).astype(np.float64) - ref)
    assert (off <= tol).all(), off.max()
    own = widen(host(call(pkg, c), c["dtype"]), c["dtype"])
    assert (np.abs(own - ref) <= tol + HALF_STEP[c["dtype"]] * (np.abs(ref) + tol) + LEAST[c["dtype"]]).all()


@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (64, "bf16"), (128, "f16"), (128, "bf16")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{len(s[0])}-L{max(s[0])}-k{max(s[1])}-{s[2]}x{s[3]}")
def test_weights(shape, d, dtype, is_tree, pkg):  # noqa: F811
    ctx, spec, hq, hkv = shape
    check(pkg, make(240 + d, ctx, spec, hq, hkv, d, dtype, is_tree))


@pytest.mark.parametrize("d", [64, 128])
def test_weights_that_round_alike(d, pkg):  # noqa: F811
    """All scores equal and values of one sign: what is lost of one weight is lost of all, and no mean evens it out."""
    c = make(250 + d, [700, 90, 2100], [3, 5, 0], 8, 2, d, "bf16")
    c["k8"][:] = 0
    c["v8"] &= 0x7f
    check(pkg, c)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("is_tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("apart", [5, 9, 60])
def test_weights_of_pages_of_very_different_scales(apart, is_tree, d, pkg):  # noqa: F811
    """Single pages 2^apart as loud as the others, whose weights are as much smaller.  Scores of up to `longest` in magnitude are
    sums of d products and two factors, off by (d + 2) 2^-24 of it, weights and their sum by that much each; what is lost to subnormals:
    2^-26 of the row's largest weighted scale per token."""
    ctx, spec = [593, 900, 2100], [6, 5, 3]
    c = make(260, ctx, spec, 8, 2, d, "bf16", is_tree)
    c["q"] = store(np.abs(widen(c["q"], "bf16")), "bf16")
    from oracle import positions as P
    for i, L in enumerate(ctx):
        page = c["bt"][i, L // 64]
        c["vs"][page] *= np.float32(2.0 ** apart)
        c["k8"][page] = P.to_e4m3(np.array([-256.0]))[0]
        c["ks"][page] = apart * np.log(2.0) / (0.8 * np.sqrt(d)) / 256.0
    ref, size = oracle(c)
    k = P.E4M3[c["k8"]] * c["ks"][..., None, None].astype(np.float64)
    longest = np.sqrt(np.nanmax((np.nan_to_num(k) ** 2).sum(-1)) * (widen(c["q"], "bf16") ** 2).sum(-1).max()) / np.sqrt(d)
    tol = (TOL + WEIGHTS + 2 * (d + 2) * 2.0 ** -24 * longest) * size + 2.0 ** -26 * max(ctx) * size.max(axis=-1, keepdims=True)
    off = np.abs(host(call(pkg, c, out_dtype=0)).astype(np.float64) - ref)
    assert (off <= tol).all(), (off / size).max()
