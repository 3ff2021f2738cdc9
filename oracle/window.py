"""CPU oracle of windowed verification attention: softmax(scale q K^T) V in float64 over the tokens a row sees, which are
the `window` up to its own position and the request's first `sinks`.

TEST INFRASTRUCTURE ONLY (see the package docstring)."""
from __future__ import annotations

import numpy as np

from workloads.verify_step import to_f64


def visible(pos: int, window: int, sinks: int) -> np.ndarray:
    """Token positions that the row at `pos` sees, ascending."""
    t = np.arange(pos + 1)
    return t[(t > pos - window) | (t < sinks)]


def hidden_tokens(ctx_len: int, n: int, window: int, sinks: int) -> np.ndarray:
    """Cached tokens that none of the request's n rows sees."""
    t = np.arange(ctx_len)
    return t[(t <= ctx_len - n - window) & (t >= sinks)]


def verify_attn_window(q, k_pages, v_pages, block_table, ctx_lens, spec_lens, *, window: int, sinks: int, dtype: str, scale=None):
    """[TQ][Hq][d] float64.  q, k_pages, v_pages as stored (dtype "f32", "f16" or bf16 bit patterns)."""
    P, Hkv, d = k_pages.shape[2], k_pages.shape[1], k_pages.shape[3]
    G = q.shape[1] // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    qd = to_f64(q, dtype)
    out = np.zeros(q.shape, np.float64)
    row = 0
    for i in range(len(spec_lens)):
        n, L = int(spec_lens[i]) + 1, int(ctx_lens[i])
        for j in range(n):
            t = visible(L - n + j, window, sinks)
            pages = block_table[i, t // P]
            k = to_f64(k_pages[pages, :, t % P], dtype)             # [T][Hkv][d]
            v = to_f64(v_pages[pages, :, t % P], dtype)
            for h in range(q.shape[1]):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (k[:, h // G] @ qd[row, h])
                    w = np.exp(s - s.max())
                    out[row, h] = (w @ v[:, h // G]) / w.sum()
            row += 1
    return out
