"""Inputs of the tests of positions and of the cache in 8 bits: ragged rows, block tables, caches, and their tensors."""
import numpy as np

from oracle.positions import to_e4m3
from workloads.verify_step import bf16_bits_to_f32, f32_to_bf16_bits

HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # of a rounding, relative
LEAST = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}       # and of what is subnormal


def store(x, dtype):
    x = np.asarray(x, np.float32)
    return f32_to_bf16_bits(x) if dtype == "bf16" else x.astype(np.float16 if dtype == "f16" else np.float32)


def dev(x, dtype=None):
    """a numpy array on the GPU; dtype "bf16" or "e4m3": of those bits"""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    if dtype == "bf16":
        t = t.view(torch.int16).view(torch.bfloat16)
    return (t.view(torch.float8_e4m3fn) if dtype == "e4m3" else t).cuda()


def host(t, dtype=None):
    """a tensor as the oracle wants it"""
    import torch
    t = t.cpu()
    if dtype == "bf16":
        return t.view(torch.int16).numpy().view(np.uint16)
    return (t.view(torch.uint8) if dtype == "e4m3" else t).numpy()


def ints(*x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def widen(x, dtype):
    return bf16_bits_to_f32(x).astype(np.float64) if dtype == "bf16" else x.astype(np.float64)


def table(rng, ctx, slack=5, width=None):
    """(block_table with -1 behind a request's pages, number of pages): distinct shuffled pages"""
    pages = [-(-int(L) // 16) for L in ctx]
    num = sum(pages) + slack
    ids, at = rng.permutation(num), 0
    out = np.full((len(ctx), width or max(pages)), -1, np.int32)
    for i, n in enumerate(pages):
        out[i, :n] = ids[at:at + n]
        at += n
    return out, num


def tree(rng, spec, width=3):
    out = []
    for k in spec:
        out += [int(rng.integers(-2, 3))] + [int(max(0, j - 1 - rng.integers(0, width))) for j in range(1, k + 1)]
    return np.array(out, np.int32)


def cache8(rng, num, hkv, d, loud=1.0):
    """(bytes, scales) of a pool as appends leave it"""
    x = rng.normal(0, loud, (num, hkv, 16, d))
    s = 2.0 ** np.ceil(np.log2(np.abs(x).max(axis=(2, 3)) / 448))
    return to_e4m3(x / s[..., None, None]), s.astype(np.float32)
