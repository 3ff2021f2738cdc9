"""CPU oracle of rotary positions and of a cache held in 8 bits (e4m3 with a scale per page and kv head), in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring)."""
from __future__ import annotations

import numpy as np

from oracle.window import visible
from workloads.verify_step import to_f64

PAGE = 16
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -100

# the value of every e4m3 byte: sign, 4 bits of exponent (bias 7), 3 of significand; no infinity, NaN where all seven are set
_CODES = np.arange(256)
_EXP, _FRAC = (_CODES >> 3) & 15, _CODES & 7
E4M3 = np.where(_EXP == 0, _FRAC / 8.0 * 2.0 ** -6, (1 + _FRAC / 8.0) * 2.0 ** (_EXP - 7.0)) * np.where(_CODES & 128, -1.0, 1.0)
E4M3[[0x7f, 0xff]] = np.nan


def to_e4m3(x) -> np.ndarray:
    """Bytes: nearest value, ties to the even code; magnitudes up to 464 (which round to 448), or not finite (NaN)."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x)
    a = np.abs(np.where(finite, x, 0.0))
    assert a.max(initial=0.0) < 464.0
    mags = E4M3[:0x7f]
    hi = np.clip(np.searchsorted(mags, a), 1, 0x7e)
    lo = hi - 1
    up = (a - mags[lo] > mags[hi] - a) | ((a - mags[lo] == mags[hi] - a) & (hi % 2 == 0))
    code = np.where(up, hi, lo).astype(np.uint8)
    return np.where(finite, code | np.where(np.signbit(x), 128, 0), 0x7f).astype(np.uint8)


def depths(parents, n: int):
    """depth of the n nodes of one request; parents outside [0, j) forced into that range, None: a chain"""
    d = [0] * n
    for j in range(1, n):
        d[j] = d[j - 1 if parents is None else min(max(int(parents[j]), 0), j - 1)] + 1
    return d


def row_positions(ctx_lens, spec_lens, parents=None):
    """(position, request, slot) of every row"""
    out, row = [], 0
    for i, (L, k) in enumerate(zip(ctx_lens, spec_lens)):
        n = int(k) + 1
        for j, dep in enumerate(depths(None if parents is None else parents[row:row + n], n)):
            out.append((int(L) - n + dep, i, int(L) - n + j))
        row += n
    return out


def _pairs(rot: int, interleaved: bool):
    f = np.arange(rot // 2)
    return (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)


def rope(x, inv_freq, ctx_lens, spec_lens, *, dtype: str, interleaved=False, attn_factor=1.0, parents=None) -> np.ndarray:
    """x [TQ][H][d] as stored; float64"""
    y = to_f64(x, dtype).copy()
    a_at, b_at = _pairs(2 * len(inv_freq), interleaved)
    for row, (p, _, _) in enumerate(row_positions(ctx_lens, spec_lens, parents)):
        # the fraction of a turn, exactly: p * freq has at most 55 bits, and long double more
        turns = np.longdouble(p) * np.asarray(inv_freq, np.float32).astype(np.longdouble) / (2 * np.longdouble("3.14159265358979323846264338327950288"))
        angle = (2 * np.pi * (turns - np.rint(turns)).astype(np.float64))
        c, s = np.cos(angle) * np.float32(attn_factor), np.sin(angle) * np.float32(attn_factor)
        a, b = y[row][:, a_at].copy(), y[row][:, b_at].copy()
        with np.errstate(invalid="ignore"):
            y[row][:, a_at], y[row][:, b_at] = a * c - b * s, b * c + a * s
    return y


def _longest2(x, rot, interleaved, attn_factor):
    """[rows][heads]: the largest squared length of a turned pair (times attn_factor) and of the other entries that are finite"""
    x = np.asarray(x, np.float64)
    a_at, b_at = _pairs(rot, interleaved)
    with np.errstate(invalid="ignore", over="ignore"):
        pairs, rest = x[..., a_at] ** 2 + x[..., b_at] ** 2, x[..., rot:] ** 2
    most = lambda v: np.where(np.isfinite(v), v, 0.0).max(axis=-1, initial=0.0)                # noqa: E731
    return np.maximum(most(pairs) * float(np.float32(attn_factor)) ** 2, most(rest))


def scale_for(most2) -> float:
    """least power of two s >= 2^-100 with most2 <= (448 s)^2"""
    s = LEAST_SCALE
    while most2 > (E4M3_MAX * s) ** 2:
        s *= 2.0
    return s


def append_scaled(k_new, v_new, inv_freq, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, *, dtype: str,
                  interleaved=False, attn_factor=1.0, parents=None):
    """New (k_pages, v_pages, k_scales, v_scales): bytes [num_pages][Hkv][16][d], float64 scales."""
    k64, v64 = to_f64(k_new, dtype), to_f64(v_new, dtype)
    rot = 0 if inv_freq is None else 2 * len(inv_freq)
    turned = k64 if inv_freq is None else rope(k_new, inv_freq, ctx_lens, spec_lens, dtype=dtype, interleaved=interleaved,
                                               attn_factor=attn_factor, parents=parents)
    out = []
    for x, raw, r, pages, scales in ((turned, k64, rot, k_pages, k_scales), (v64, v64, 0, v_pages, v_scales)):
        pages, scales = pages.copy(), np.asarray(scales, np.float64).copy()
        most2, row = _longest2(raw, r, interleaved, attn_factor), 0
        for i, (L, k) in enumerate(zip(ctx_lens, spec_lens)):
            L, n = int(L), int(k) + 1
            for p in range((L - n) // PAGE, (L - 1) // PAGE + 1):
                lo, hi, page = max(L - n, p * PAGE), min(L, p * PAGE + PAGE), int(block_table[i][p])
                rows = slice(row + lo - (L - n), row + hi - (L - n))
                for h in range(pages.shape[1]):
                    s = scale_for(most2[rows, h].max())
                    if lo > p * PAGE:
                        s = max(s, scales[page, h])
                        if s != scales[page, h]:
                            kept = pages[page, h, :lo - p * PAGE]
                            pages[page, h, :lo - p * PAGE] = to_e4m3(E4M3[kept] * (scales[page, h] / s))
                    scales[page, h] = s
                    pages[page, h, lo - p * PAGE:hi - p * PAGE] = to_e4m3(x[rows, h] / s)
            row += n
        out.append((pages, scales))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def compact_path_scaled(pages, scales, block_table, ctx_lens, spec_lens, out_path, out_accept_len):
    """New (pages, scales) of K or of V."""
    pages, scales = pages.copy(), np.asarray(scales, np.float64).copy()
    for i, (L, k, a) in enumerate(zip(ctx_lens, spec_lens, out_accept_len)):
        base = int(L) - int(k) - 1
        moves = [(base + int(out_path[i][j]), base + 1 + j) for j in range(int(a))]
        where = lambda t: (int(block_table[i][t // PAGE]), t % PAGE)                           # noqa: E731
        for h in range(pages.shape[1]):
            value = {t: (pages[where(t)[0], h, where(t)[1]].copy(), scales[where(t)[0], h]) for t in range(base // PAGE * PAGE, int(L))}
            new = {}
            for src, dst in moves:
                page = where(dst)[0]
                new[page] = max(new.get(page, scales[page, h]), value[src][1])
            moved = {dst: value[src] for src, dst in moves}
            for t in range(base // PAGE * PAGE, base + 1 + len(moves)):
                page, slot = where(t)
                byte, s = moved.get(t, value[t])
                s1 = new.get(page, scales[page, h])
                pages[page, h, slot] = byte if s == s1 else to_e4m3(E4M3[byte] * (s / s1))
            for page, s in new.items():
                scales[page, h] = s
    return pages, scales


def verify_attn_scaled(q, k_pages, v_pages, k_scales, v_scales, block_table, ctx_lens, spec_lens, *, dtype: str, parents=None, scale=None):
    """[TQ][Hq][d] float64"""
    Hkv, d = k_pages.shape[1], k_pages.shape[3]
    G = q.shape[1] // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    qd, out, row = to_f64(q, dtype), np.zeros(q.shape, np.float64), 0
    for i, (L, spec) in enumerate(zip(ctx_lens, spec_lens)):
        L, n = int(L), int(spec) + 1
        t = np.arange(L)
        pages = np.asarray(block_table[i])[t // PAGE]
        with np.errstate(invalid="ignore"):
            k = E4M3[k_pages[pages, :, t % PAGE]] * np.asarray(k_scales, np.float64)[pages][..., None]      # [T][Hkv][d]
            v = E4M3[v_pages[pages, :, t % PAGE]] * np.asarray(v_scales, np.float64)[pages][..., None]
        up = [0] * n
        for j in range(1, n):
            up[j] = j - 1 if parents is None else min(max(int(parents[row + j]), 0), j - 1)
        for j in range(n):
            if parents is None:
                sees = visible(L - n + j, L, 0)
            else:
                chain, u = [j], j
                while u:
                    u = up[u]
                    chain.append(u)
                sees = np.concatenate([np.arange(L - n), L - n + np.array(sorted(chain))])
            for h in range(q.shape[1]):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (k[sees, h // G] @ qd[row + j, h])
                    w = np.exp(s - s.max())
                    out[row + j, h] = (w @ v[sees, h // G]) / w.sum()
        row += n
    return out
