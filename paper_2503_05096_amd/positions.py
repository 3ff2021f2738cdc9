"""Frequencies of rotary positions: what rope and kv_append_rope take as inv_freq and attn_factor."""
from __future__ import annotations

import math
from typing import Optional, Tuple


def rope_frequencies(rot_dim: int, *, base: float = 10000.0, scaling: Optional[dict] = None, device=None) -> Tuple[object, float]:
    """(inv_freq [rot_dim / 2] float32, attn_factor): base^(-2f / rot_dim), for contexts longer than the model was trained on changed
    by `scaling`, a dict with "kind" and "factor" (the longer context over the trained one):

      "linear"       every frequency divided by factor, positions are squeezed (position interpolation: Chen et al. 2023,
                     arXiv:2306.15595)
      "base"         base times factor^(rot_dim / (rot_dim - 2)): the fastest pair stays, the slowest is divided by factor (NTK-aware
                     scaling: Peng et al. 2023, arXiv:2309.00071, section 3.1)
      "wavelengths"  divided by factor where a turn takes more than trained / low tokens, kept where it takes fewer than
                     trained / high, blended between (trained: the trained context; low, high: 1 and 4; published with the
                     Llama 3.1 models)
      "ramp"         divided by factor where the trained context has fewer than slow turns, kept where it has more than
                     fast, blended linearly in the pair's number between (trained; slow, fast: 1 and 32); attn_factor is
                     0.1 ln(factor) + 1 unless given as "attn_factor" (YaRN: Peng et al. 2023, sections 3.2 to 3.4)

    Worked out in 64 bits on the host, rounded once."""
    import torch
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rope_frequencies(rot_dim) is even and at least 2")
    if not base > 0:
        raise ValueError("rope_frequencies(base=...) is more than 0")
    s = dict(scaling or {"kind": None})
    kind, factor = s.pop("kind"), float(s.pop("factor", 1.0))
    if not factor > 0:
        raise ValueError("rope_frequencies: the factor of a scaling is more than 0")
    half, gain = rot_dim // 2, 1.0
    if kind == "base":
        if rot_dim == 2:
            raise ValueError("rope_frequencies: a single pair has no slowest frequency to fix a base by")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    freq = [base ** (-2.0 * f / rot_dim) for f in range(half)]
    if kind in (None, "base"):
        pass
    elif kind == "linear":
        freq = [x / factor for x in freq]
    elif kind == "wavelengths":
        trained, low, high = float(s.pop("trained")), float(s.pop("low", 1.0)), float(s.pop("high", 4.0))
        if not 0 < low < high:
            raise ValueError("rope_frequencies: 0 < low < high")
        turns = [trained * x / (2.0 * math.pi) for x in freq]
        keep = [min(max((t - low) / (high - low), 0.0), 1.0) for t in turns]
        freq = [x * (k + (1.0 - k) / factor) for x, k in zip(freq, keep)]
    elif kind == "ramp":
        trained, slow, fast = float(s.pop("trained")), float(s.pop("slow", 1.0)), float(s.pop("fast", 32.0))
        if not 0 < slow < fast or not base > 1:
            raise ValueError("rope_frequencies: 0 < slow < fast, and a base above 1")
        pair = lambda turns: half * math.log(trained / (2.0 * math.pi * turns)) / math.log(base)        # noqa: E731
        # The ramp ends at whole pairs, outwards.  Its upper end is cut at the number of entries, not of pairs, as in the models that were
        # trained with this scaling: an end behind the last pair is part of their slope.  Ends that meet make a step (0.001 for the 0 between).
        lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot_dim - 1)
        keep = [1.0 - min(max((f - lo) / max(hi - lo, 0.001), 0.0), 1.0) for f in range(half)]
        freq = [x * (k + (1.0 - k) / factor) for x, k in zip(freq, keep)]
        gain = float(s.pop("attn_factor", 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0))
    else:
        raise ValueError(f"rope_frequencies: no scaling {kind!r}")
    if s:
        raise ValueError(f"rope_frequencies: what is {sorted(s)}?")
    return torch.tensor(freq, dtype=torch.float64).float().to("cpu" if device is None else device), gain
