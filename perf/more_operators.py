"""Operators of a cache held in 8 bits and of the positions that go into it, measured one call a pass.

  rope     rope: query rows turned by the angles of their positions
  append   kv_append_rope: queries turned, keys turned and written into the paged cache with the values, 16 bits or fp32
  append8  the same into a cache of e4m3 with a power-of-two scale for each page and kv head
  attn8    verify_attn over such a cache

Rows are ragged as in the verification step: request i has spec_lens[i] + 1 of them, the last of its ctx_lens[i] tokens; row
j stands at position ctx_lens[i] - n_i + j, in a draft tree (width > 1) at the root's position plus its depth.

`own` false: the same in elementary torch operations, in 32 bits, angles and scales in 64.  A case fixes the sizes and the
multiset of lengths; the seed decides who gets which, where the pages lie, and the values.
"""
import math
import random

import torch

own = False

PAGE = 16
_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_E4M3 = torch.float8_e4m3fn
_E4M3_MAX = 448.0
_LEAST_EXPONENT = -100          # of a scale


# --------------------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------------------
def _rope(name, dtype, batch, ctx_lo, ctx_hi, spec_lo, spec_hi, heads, d, rot, interleaved, base, width=1):
    return dict(name=name, kind="rope", dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi,
                hq=heads, hkv=0, d=d, rot=rot, interleaved=interleaved, base=base, factor=1.0, gain=1.0, width=width)


def _append(name, kind, dtype, batch, ctx_lo, ctx_hi, spec_lo, spec_hi, hq, hkv, d, rot, interleaved, base, factor=1.0, gain=1.0,
            width=1):
    return dict(name=name, kind=kind, dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi,
                hq=hq, hkv=hkv, d=d, rot=rot, interleaved=interleaved, base=base, factor=factor, gain=gain, width=width)


def _attn8(name, dtype, batch, ctx_lo, ctx_hi, spec_lo, spec_hi, hq, hkv, d, width=1):
    return dict(name=name, kind="attn8", dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi,
                hq=hq, hkv=hkv, d=d, width=width)


def listed():
    return [
        # one token of one user, far into a conversation: latency alone
        _rope("rope-one-token", "bf16", 1, 60000, 60000, 0, 0, 32, 128, 128, False, 500000.0),
        # prompts of a model that turns the first half of its heads, neighbours paired
        _rope("rope-prompts-partial", "f16", 8, 256, 4096, 255, 4095, 32, 128, 64, True, 10000.0),
        # a unit-sized fp32 batch as in development and in accuracy checks (benchmark config 1's heads)
        _append("append-f32-tiny", "append", "f32", 4, 128, 512, 1, 4, 8, 8, 64, 64, False, 10000.0),
        # the verification step of the headline batch (config 3's heads), 16-bit cache
        _append("append-step", "append", "bf16", 128, 128, 2048, 0, 6, 32, 8, 128, 128, False, 500000.0),
        # ragged prompts into the cache, positions stretched for a long context
        _append("append-prompts", "append", "bf16", 16, 100, 4000, 99, 3999, 32, 8, 128, 128, False, 500000.0, 8.0, 1.2),
        # the verification step of the headline batch into a cache of 8 bits
        _append("append8-step", "append8", "bf16", 128, 128, 2048, 0, 6, 32, 8, 128, 128, False, 500000.0),
        # draft trees of a small batch into a cache of 8 bits
        _append("append8-trees", "append8", "bf16", 16, 200, 1500, 20, 60, 32, 8, 128, 128, False, 10000.0, width=3),
        # ragged prompts into a cache of 8 bits, the 70B layout (config 4's heads)
        _append("append8-prompts", "append8", "bf16", 16, 100, 4000, 99, 3999, 64, 8, 128, 128, False, 500000.0),
        # one interactive user far into a long conversation
        _attn8("attn8-one-request", "bf16", 1, 60000, 60000, 5, 5, 32, 8, 128),
        # the headline batch (config 3)
        _attn8("attn8-gqa", "bf16", 128, 128, 4096, 0, 6, 32, 8, 128),
        # the 70B layout on long contexts: many query rows per kv head (config 4's heads), the largest
        _attn8("attn8-gqa-long", "bf16", 64, 8192, 32768, 0, 5, 64, 8, 128),
        # a 1B-sized model with 64-wide heads, draft trees
        _attn8("attn8-d64-trees", "f16", 64, 256, 4096, 3, 12, 32, 8, 64, width=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (query heads, kv heads, head dim): the configurations' head layouts and those between them
_HEADS = ((32, 32, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 2, 128), (15, 3, 128), (8, 8, 64), (32, 8, 64), (14, 2, 64))
_MOST_ROWS_BYTES = 2e8        # new rows of one pass, read
_MOST_KV_BYTES = 1e9          # cached K and V of one pass
_MOST_SCORES = 8e8            # products of a query row with a key


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(("rope", "append", "append", "append8", "append8", "attn8", "attn8", "attn8"))
    hq, hkv, d = rng.choice(_HEADS)
    width = rng.choice((1, 1, 1, rng.randint(2, 4)))
    if kind == "attn8":
        dtype = rng.choice(("bf16", "bf16", "f16"))
        spec_hi = rng.randint(0, 8) if width == 1 else _log(rng, 2, 63)
        spec_lo = rng.randint(0, spec_hi)
        ctx_hi = _log(rng, max(24, spec_hi + 1), 65536)
        ctx_lo = max(spec_hi + 1, int(ctx_hi * rng.uniform(0.05, 1.0)))
        ctx_hi = max(ctx_hi, ctx_lo)
        batch = _log(rng, 1, max(1, min(256, int(_MOST_KV_BYTES / (hkv * d * (ctx_lo + ctx_hi))),
                                        int(_MOST_SCORES / (hq * (spec_hi + 1) * ctx_hi)))))
        return dict(kind=kind, dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi, hq=hq,
                    hkv=hkv, d=d, width=width)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    prompts = width == 1 and rng.random() < 0.4
    if prompts:
        spec_hi = _log(rng, 16, 4095)
        spec_lo = rng.randint(0, spec_hi)
        ctx_lo = ctx_hi = spec_hi + 1 + rng.choice((0, rng.randint(0, 2000)))
    else:
        spec_hi = rng.randint(0, 8) if width == 1 else _log(rng, 2, 63)
        spec_lo = rng.randint(0, spec_hi)
        ctx_hi = _log(rng, max(24, spec_hi + 1), 4096)
        ctx_lo = max(spec_hi + 1, int(ctx_hi * rng.uniform(0.05, 1.0)))
        ctx_hi = max(ctx_hi, ctx_lo)
    row = (hq + 2 * hkv) * d * _SIZE[dtype]
    batch = _log(rng, 1, max(1, min(256, int(_MOST_ROWS_BYTES / (row * (1 + (spec_lo + spec_hi) / 2))),
                                    int(_MOST_KV_BYTES / (hkv * d * 2 * (ctx_lo + ctx_hi))))))
    rot = rng.choice((d, d, d // 2, 2 * rng.randint(1, d // 2)))
    if kind == "rope":
        hkv = 0
    return dict(kind=kind, dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi, hq=hq, hkv=hkv,
                d=d, rot=rot, interleaved=rng.random() < 0.4, base=rng.choice((10000.0, 500000.0, 1000000.0)),
                factor=rng.choice((1.0, 1.0, 4.0, 8.0)), gain=rng.choice((1.0, 1.0, 1.2)), width=width)


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
class _State:
    pass


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _quantiles(lo, hi, n):
    return [lo + int((hi - lo) * (i + 0.5) / n) for i in range(n)]


def _spec_list(c):
    lo, hi, n = c["spec_lo"], c["spec_hi"], c["batch"]
    return [lo + min(hi - lo, int((hi - lo + 1) * (i + 0.5) / n)) for i in range(n)]


def _ctx_list(c, spec):
    """Context lengths; those of prompts, which are longer than the shortest context, follow the prompts' own."""
    ctx = _quantiles(c["ctx_lo"], c["ctx_hi"], c["batch"])
    return [max(L, k + 1) for L, k in zip(ctx, spec)]


def _parents(spec, width, r):
    """A tree for every request: a draft hangs on the most recent node with fewer than `width` children, or on any such node."""
    out = []
    for k in spec:
        children, row = [0] * (k + 1), [0]
        for j in range(1, k + 1):
            open_ = [u for u in range(j) if children[u] < width]
            u = open_[-1] if r.random() < 0.5 else r.choice(open_)
            children[u] += 1
            row.append(u)
        out += row
    return _ints(out)


def _cache8(pages, hkv, d, gen):
    """Pages of 8 bits with their scales, as earlier steps have left them: keys with a few large channels, values without."""
    loud = 1.0 + 5.0 * (torch.rand(hkv, 1, d, generator=gen, device="cuda") > 0.97)
    made = []
    for lean in (loud, None):
        x8 = torch.empty(pages, hkv, PAGE, d, dtype=_E4M3, device="cuda")
        scales = torch.empty(pages, hkv, device="cuda")
        part = max(1, (1 << 26) // (hkv * PAGE * d))
        for at in range(0, pages, part):
            x = torch.empty(min(part, pages - at), hkv, PAGE, d, device="cuda").normal_(0.0, 1.0, generator=gen)
            if lean is not None:
                x *= lean
            s = torch.exp2(torch.ceil(torch.log2(x.abs().amax(dim=(2, 3)) / _E4M3_MAX)))
            x8[at:at + part] = (x / s[:, :, None, None]).to(_E4M3)
            scales[at:at + part] = s
        made += [x8, scales]
    return made


def prepare(case, seed):
    s, c = _State(), case
    s.case = c
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    r = random.Random("inputs %d" % seed)
    spec = _spec_list(c)
    ctx = _ctx_list(c, spec)
    both = list(zip(ctx, spec))
    r.shuffle(both)
    if c["ctx_lo"] > c["spec_hi"]:              # (any context takes any draft length)
        r.shuffle(spec)
        both = [(L, k) for (L, _), k in zip(both, spec)]
    s.ctx_list, s.spec_list = [L for L, _ in both], [k for _, k in both]
    s.ctx_lens, s.spec_lens = _ints(s.ctx_list), _ints(s.spec_list)
    s.parents = _parents(s.spec_list, c["width"], r) if c["width"] > 1 else None
    rows, hq, hkv, d, dtype = sum(s.spec_list) + len(spec), c["hq"], c["hkv"], c["d"], _TORCH[c["dtype"]]
    # what a model's projection leaves: a token's queries, keys and values side by side in one row
    s.qkv = torch.empty(rows, (hq + 2 * hkv) * d, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen)
    s.q = s.qkv[:, :hq * d].unflatten(1, (hq, d))
    if c["kind"] != "attn8":
        turns = torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"]
        s.inv_freq = (c["base"] ** -turns / c["factor"]).float().cuda()
    if c["kind"] == "rope":
        return s
    s.k = s.qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    s.v = s.qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
    pages = [-(-L // PAGE) for L in s.ctx_list]
    ids = list(range(max(1, math.ceil(1.1 * sum(pages)))))
    r.shuffle(ids)
    table, at = torch.full((len(pages), max(pages)), -1, dtype=torch.int32), 0
    for i, n in enumerate(pages):
        table[i, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
        at += n
    s.block_table = table.cuda()
    if c["kind"] == "append":
        kv = (len(ids), hkv, PAGE, d)
        s.k_pages, s.v_pages = (torch.empty(kv, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen) for _ in range(2))
        return s
    s.k_pages, s.k_scales, s.v_pages, s.v_scales = _cache8(len(ids), hkv, d, gen)
    if c["kind"] == "append8":                  # now and then a token is louder than its page so far
        s.qkv *= torch.exp2(2.0 * (torch.rand(rows, 1, generator=gen, device="cuda") > 0.8)).to(dtype)
    else:
        s.q = s.q.contiguous()
        del s.qkv, s.k, s.v
    return s


# --------------------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------------------
def _rows(s):
    """Of every row: its request and its index there; the requests' first rows."""
    n = s.spec_lens.long() + 1
    end = n.cumsum(0)
    row = torch.arange(s.q.shape[0], device=n.device)
    owner = torch.searchsorted(end, row, right=True)
    return owner, row - (end - n)[owner], end - n


def _sees(s, owner, local):
    """[B][n][n]: whether a request's second node is the first or one of its ancestors."""
    most = s.case["spec_hi"] + 1
    step = torch.zeros(s.case["batch"], most, most, device=owner.device)
    drafts = local > 0
    step[owner[drafts], local[drafts], s.parents.long()[drafts]] = 1.0
    return torch.linalg.matrix_power(step + torch.eye(most, device=owner.device), most) > 0


def _positions(s):
    owner, local, _ = _rows(s)
    depth = local if s.parents is None else _sees(s, owner, local)[owner, local].sum(-1) - 1
    return (s.ctx_lens.long() - s.spec_lens.long() - 1)[owner] + depth


def _turned(x, position, s):
    """x [rows][heads][d] turned by the angles of its rows' positions, in 32 bits."""
    c = s.case
    half = c["rot"] // 2
    angle = position.double()[:, None] * s.inv_freq.double()
    cos, sin = (torch.cos(angle) * c["gain"]).float()[:, None], (torch.sin(angle) * c["gain"]).float()[:, None]
    x = x.float()
    y = x.clone()
    if c["interleaved"]:
        a, b = x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2]
        y[..., 0:c["rot"]:2], y[..., 1:c["rot"]:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:c["rot"]]
        y[..., :half], y[..., half:c["rot"]] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_append(s, c):
    owner, local, _ = _rows(s)
    position = _positions(s)
    slot = (s.ctx_lens.long() - s.spec_lens.long() - 1)[owner] + local
    page = s.block_table.long()[owner, slot // PAGE]
    s.k_pages[page, :, slot % PAGE] = _turned(s.k, position, s).to(s.k.dtype)
    s.v_pages[page, :, slot % PAGE] = s.v
    return {"q": _turned(s.q, position, s).to(s.q.dtype), "k_pages": s.k_pages, "v_pages": s.v_pages}


def _longest(x, s):
    """[rows][heads], 64 bits: the largest squared length of a key's pairs, which turning keeps, and of its other entries."""
    c, x = s.case, x.double()
    half, rest = c["rot"] // 2, x[..., c["rot"]:].square()
    a, b = (x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2]) if c["interleaved"] else (x[..., :half], x[..., half:c["rot"]])
    gain = torch.tensor(c["gain"], dtype=torch.float32).double().item()
    most = (a.square() + b.square()).amax(-1) * (gain * gain)
    return torch.maximum(most, rest.amax(-1)) if c["rot"] < c["d"] else most


def _scale_for(most):
    """The least power of two s with most <= (448 s)^2; 448^2 = 1.53125 * 2^17."""
    fraction, exponent = torch.frexp(most)
    exponent = exponent - 18                                    # most = 2 fraction 2^17 2^exponent
    up = torch.where(exponent % 2 == 0, (2 * fraction > 1.53125).int(), 1)
    e = torch.div(exponent, 2, rounding_mode="floor") + up
    return torch.exp2(torch.where(most > 0, e, _LEAST_EXPONENT).clamp(min=_LEAST_EXPONENT).float())


def _plain_append8(s, c):
    owner, local, start = _rows(s)
    position = _positions(s)
    q = _turned(s.q, position, s).to(s.q.dtype)
    # the pages that get new tokens: [B][S], with their 16 slots
    L, first = s.ctx_lens.long(), s.ctx_lens.long() - s.spec_lens.long() - 1
    index = first[:, None] // PAGE + torch.arange((c["spec_hi"] + PAGE - 1) // PAGE + 1, device=L.device)
    b, at = (index * PAGE < L[:, None]).nonzero(as_tuple=True)
    index = index[b, at]
    page = s.block_table.long()[b, index]
    token = index[:, None] * PAGE + torch.arange(PAGE, device=L.device)
    new, kept = (token >= first[b, None]) & (token < L[b, None]), token < first[b, None]
    row = (start[b, None] + token - first[b, None]).clamp(min=0, max=s.q.shape[0] - 1)
    out = {"q": q}
    for name, x, most in (("k", _turned(s.k, position, s), _longest(s.k, s)), ("v", s.v.float(), s.v.double().square().amax(-1))):
        pages, scales = getattr(s, name + "_pages"), getattr(s, name + "_scales")
        need = _scale_for(torch.where(new[..., None], most[row], 0.0).amax(1))                       # [pages][Hkv]
        old = scales[page]
        scale = torch.where(kept.any(1)[:, None], torch.maximum(old, need), need)
        values = torch.where(new[..., None, None], x[row], 0.0).transpose(1, 2) / scale[:, :, None, None]
        before = pages.view(torch.uint8)[page]
        again = before.view(_E4M3).float() * (old / scale)[:, :, None, None]
        both = torch.where(new[:, None, :, None], values.to(_E4M3).view(torch.uint8),
                           torch.where(kept[:, None, :, None], again.to(_E4M3).view(torch.uint8), before))
        pages.view(torch.uint8)[page] = both
        scales[page] = scale
        out |= {name + "_pages": pages, name + "_scales": scales}
    return out


def _plain_attn8(s, c):
    B, hkv, d, G, most = c["batch"], c["hkv"], c["d"], c["hq"] // c["hkv"], c["spec_hi"] + 1
    owner, local, start = _rows(s)
    n, L = s.spec_lens.long() + 1, s.ctx_lens.long()
    dev = L.device
    table = torch.where(torch.arange(s.block_table.shape[1], device=dev) * PAGE < L[:, None], s.block_table.long(), 0)
    T = table.shape[1] * PAGE
    k = s.k_pages.view(torch.uint8)[table].view(_E4M3).float() * s.k_scales[table][..., None, None]         # [B][pages][Hkv][16][d]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, hkv, d, T)
    t, j = torch.arange(T, device=dev), torch.arange(most, device=dev)
    q = s.q[start[:, None] + torch.minimum(j, n[:, None] - 1)].float().view(B, most, hkv, G, d).permute(0, 2, 1, 3, 4)
    score = torch.matmul(q.reshape(B, hkv, most * G, d), k).view(B, hkv, most, G, T) * d ** -0.5
    del k
    first = (L - n)[:, None]
    sees = (t <= first[:, :, None] + j[:, None]) & (t < L[:, None, None])                                   # [B][n][T]
    if s.parents is not None:
        new = (t - first).clamp(min=0, max=most - 1)
        sees &= (t < first)[:, None] | _sees(s, owner, local).gather(2, new[:, None].expand(-1, most, -1))
    score = score.masked_fill(~sees[:, None, :, None], float("-inf"))
    weight = torch.exp(score - score.amax(dim=-1, keepdim=True))
    del score
    total = weight.sum(dim=-1, keepdim=True)
    v = s.v_pages.view(torch.uint8)[table].view(_E4M3).float() * s.v_scales[table][..., None, None]
    v = v.permute(0, 2, 1, 3, 4).reshape(B, hkv, T, d)
    out = torch.matmul(weight.view(B, hkv, most * G, T), v).view(B, hkv, most, G, d) / total
    return {"out": out.permute(0, 2, 1, 3, 4).reshape(B, most, c["hq"], d)[owner, local].to(s.q.dtype)}


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------
def _own(s, c):
    import paper_2503_05096_amd as pkg
    if c["kind"] == "rope":
        return {"q": pkg.rope(s.q, s.inv_freq, s.ctx_lens, s.spec_lens, max_spec_len=c["spec_hi"], interleaved=c["interleaved"],
                              attn_factor=c["gain"], parents=s.parents)}
    if c["kind"] == "append":
        q = pkg.kv_append_rope(s.q, s.k, s.v, s.inv_freq, s.k_pages, s.v_pages, s.block_table, s.ctx_lens, s.spec_lens,
                               max_spec_len=c["spec_hi"], interleaved=c["interleaved"], attn_factor=c["gain"], parents=s.parents)
        return {"q": q, "k_pages": s.k_pages, "v_pages": s.v_pages}
    if c["kind"] == "append8":
        q = pkg.kv_append_rope(s.q, s.k, s.v, s.inv_freq, s.k_pages, s.v_pages, s.block_table, s.ctx_lens, s.spec_lens,
                               max_spec_len=c["spec_hi"], k_scales=s.k_scales, v_scales=s.v_scales, interleaved=c["interleaved"],
                               attn_factor=c["gain"], parents=s.parents)
        return {"q": q, "k_pages": s.k_pages, "k_scales": s.k_scales, "v_pages": s.v_pages, "v_scales": s.v_scales}
    return {"out": pkg.verify_attn(s.q, s.k_pages, s.v_pages, s.block_table, s.ctx_lens, s.spec_lens, max_spec_len=c["spec_hi"],
                                   k_scales=s.k_scales, v_scales=s.v_scales, parents=s.parents)}


def run(s):
    c = s.case
    if own:
        return _own(s, c)
    if c["kind"] == "rope":
        return {"q": _turned(s.q, _positions(s), s).to(s.q.dtype)}
    return {"append": _plain_append, "append8": _plain_append8, "attn8": _plain_attn8}[c["kind"]](s, c)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------
def work(c):
    spec = _spec_list(c)
    ctx, rows, hq, hkv, d = _ctx_list(c, spec), sum(spec) + len(spec), c["hq"], c["hkv"], c["d"]
    if c["kind"] == "attn8":
        n = rows / len(spec)
        pages = sum(-(-L // PAGE) for L in ctx)
        return {"bytes": int(sum(ctx) * 2 * hkv * d + pages * (4 + 8 * hkv) + 2 * rows * hq * d * _SIZE[c["dtype"]]),
                "flops": int(4 * d * hq * n * sum(L - (n - 1) / 2 for L in ctx))}
    size = _SIZE[c["dtype"]]
    kept = size if c["kind"] == "append" else 1
    nbytes = rows * d * (2 * hq * size + 2 * hkv * (size + kept)) + 2 * c["rot"] + 8 * len(spec)
    return {"bytes": nbytes, "flops": 3 * rows * (hq + hkv) * c["rot"]}


# --------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------
def _exact_positions(s):
    where, at = [], 0
    parents = s.parents.tolist() if s.parents is not None else None
    for L, k in zip(s.ctx_list, s.spec_list):
        depth = [0]
        for j in range(1, k + 1):
            depth.append(j if parents is None else depth[parents[at + j]] + 1)
        where += [L - k - 1 + x for x in depth]
        at += k + 1
    return torch.tensor(where, dtype=torch.float64, device=s.q.device)


def _exact_turned(x, s):
    c = s.case
    z = x.double()
    first = range(0, c["rot"], 2) if c["interleaved"] else range(c["rot"] // 2)
    second = range(1, c["rot"], 2) if c["interleaved"] else range(c["rot"] // 2, c["rot"])
    first, second = torch.tensor(first, device=z.device), torch.tensor(second, device=z.device)
    angle = torch.outer(_exact_positions(s), s.inv_freq.double())[:, None, :]
    pair = torch.complex(z[..., first], z[..., second]) * torch.polar(torch.full_like(angle, c["gain"]), angle)
    return z.index_copy(-1, first, pair.real).index_copy(-1, second, pair.imag)


def _nearest8(x):
    """x rounded to the nearest e4m3 value, ties to even; |x| <= 448."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(x / step) * step


def _exact_append8(s, c):
    out = {"q": _exact_turned(s.q, s)}
    table = s.block_table.tolist()
    for name, x in (("k", _exact_turned(s.k, s)), ("v", s.v.double())):
        pages, scales = getattr(s, name + "_pages").double(), getattr(s, name + "_scales").double()
        # a pair's length, not its turned entries, decides the scale
        size = x.abs()
        if name == "k":
            half, rot = c["rot"] // 2, c["rot"]
            raw = s.k.double()
            a, b = (raw[..., 0:rot:2], raw[..., 1:rot:2]) if c["interleaved"] else (raw[..., :half], raw[..., half:rot])
            size = torch.cat([torch.hypot(a, b) * c["gain"], raw[..., rot:].abs()], dim=-1)
        size = size.amax(-1)
        at = 0
        for i, (L, k) in enumerate(zip(s.ctx_list, s.spec_list)):
            first = L - k - 1
            for p in range(first // PAGE, (L - 1) // PAGE + 1):
                lo, hi, page = max(first, p * PAGE), min(L, p * PAGE + PAGE), table[i][p]
                most = size[at + lo - first:at + hi - first].amax(0)
                scale = torch.exp2(torch.ceil(torch.log2((most / _E4M3_MAX).clamp(min=2.0 ** _LEAST_EXPONENT))))
                if lo > p * PAGE:
                    scale = torch.maximum(scale, scales[page])
                    pages[page, :, :lo - p * PAGE] = _nearest8(pages[page, :, :lo - p * PAGE] * (scales[page] / scale)[:, None, None])
                scales[page] = scale
                pages[page, :, lo - p * PAGE:hi - p * PAGE] = _nearest8(x[at + lo - first:at + hi - first] / scale[:, None]).transpose(0, 1)
            at += k + 1
        out |= {name + "_pages": pages, name + "_scales": scales}
    return out


def _exact_attn8(s, c):
    G, d = c["hq"] // c["hkv"], c["d"]
    out = torch.empty(s.q.shape, dtype=torch.float64, device=s.q.device)
    parents = s.parents.tolist() if s.parents is not None else None
    at = 0
    for i, (L, k) in enumerate(zip(s.ctx_list, s.spec_list)):
        page = s.block_table[i, :-(-L // PAGE)].long()
        keys, values = (p.view(torch.uint8)[page].view(_E4M3).double() * z[page].double()[..., None, None]
                        for p, z in ((s.k_pages, s.k_scales), (s.v_pages, s.v_scales)))
        keys, values = (x.transpose(0, 1).reshape(c["hkv"], -1, d)[:, :L] for x in (keys, values))            # [Hkv][L][d]
        hidden = torch.ones(k + 1, k + 1, dtype=torch.bool)
        for j in range(k + 1):
            if j:
                hidden[j] = hidden[j - 1 if parents is None else parents[at + j]]
            hidden[j, j] = False
        q = s.q[at:at + k + 1].double().view(k + 1, c["hkv"], G, d).permute(1, 0, 2, 3).reshape(c["hkv"], -1, d)
        score = (torch.matmul(q, keys.transpose(1, 2).contiguous()) / math.sqrt(d)).view(c["hkv"], k + 1, G, L)
        score[..., L - k - 1:].masked_fill_(hidden.to(out.device)[:, None], -math.inf)
        p = torch.exp(score - torch.logsumexp(score, dim=-1, keepdim=True)).view(c["hkv"], -1, L)
        o = torch.matmul(p, values.contiguous()).view(c["hkv"], k + 1, G, d)
        out[at:at + k + 1] = o.permute(1, 0, 2, 3).reshape(k + 1, c["hq"], d)
        at += k + 1
    return {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return {"q": _exact_turned(s.q, s)}
    if case["kind"] == "attn8":
        return _exact_attn8(s, case)
    if case["kind"] == "append8":
        return _exact_append8(s, case)
    k, v, at = s.k_pages.double(), s.v_pages.double(), 0
    turned = _exact_turned(s.k, s)
    for i, (L, n) in enumerate(zip(s.ctx_list, s.spec_list)):
        t = torch.arange(L - n - 1, L, device=k.device)
        page = s.block_table[i].long()[t // PAGE]
        k[page, :, t % PAGE], v[page, :, t % PAGE] = turned[at:at + n + 1], s.v[at:at + n + 1].double()
        at += n + 1
    return {"q": _exact_turned(s.q, s), "k_pages": k, "v_pages": v}
