"""Operators of a cache that stays bounded, measured one call a pass: windowed verification attention, and the pages behind it.

  attn     verify_attn with a sliding window and first tokens that stay visible (sinks), over a block table with holes where
           the pages between the sinks and the window have been given back
  copy     kv_copy_pages: pairs of pages of all layers, source to destination
  remap    kv_remap: the block table of the next batch: rows dropped, forked, reordered and grown, pages behind a window
           given back, free ones handed out, the pairs that have to be copied named
  compact  kv_compact_pages: used pages to the front of the pool

`own` false: the same in elementary torch operations, in 32 bits.  A case fixes the sizes and the multiset of lengths; the
seed decides who gets which, where the pages lie, and the values.
"""
import math
import random

import torch

own = False

PAGE = 16
_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# --------------------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------------------
def _attn(name, dtype, batch, ctx_lo, ctx_hi, spec_lo, spec_hi, hq, hkv, d, window, sinks):
    return dict(name=name, kind="attn", dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi,
                hq=hq, hkv=hkv, d=d, window=window, sinks=sinks)


def _copy(name, dtype, pairs, padding, layers, hkv, d):
    return dict(name=name, kind="copy", dtype=dtype, pairs=pairs, padding=padding, layers=layers, hkv=hkv, d=d)


def _remap(name, mode, old_batch, batch, ctx_lo, ctx_hi, grow, shared, window, sinks, room):
    return dict(name=name, kind="remap", mode=mode, old_batch=old_batch, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, grow=grow,
                shared=shared, window=window, sinks=sinks, room=room)


def _compact(name, num_pages, used, batch):
    return dict(name=name, kind="compact", num_pages=num_pages, used=used, batch=batch)


def listed():
    return [
        # the smallest attention: a unit-sized fp32 batch as in development and in accuracy checks (benchmark config 1)
        _attn("window-f32-tiny", "f32", 4, 128, 512, 1, 4, 8, 8, 64, 100, 3),
        # one interactive user far into a long conversation: nothing in the batch to hide latency behind
        _attn("window-one-request", "bf16", 1, 60000, 60000, 5, 5, 32, 8, 128, 2048, 4),
        # a multi-head model in fp16 with a short window and no sinks
        _attn("window-mha-f16", "f16", 32, 256, 2048, 0, 8, 32, 32, 128, 128, 0),
        # the headline batch (config 3) with a window of a quarter of its longest context
        _attn("window-gqa", "bf16", 128, 128, 4096, 0, 6, 32, 8, 128, 1024, 4),
        # a 70B layout on contexts far beyond the window: many query rows per kv head (config 4's heads), the largest
        _attn("window-gqa-long", "bf16", 64, 8192, 32768, 0, 5, 64, 8, 128, 4096, 16),
        # a 1B-sized model with 64-wide heads, odd window and sinks
        _attn("window-d64", "bf16", 64, 256, 4096, 0, 6, 32, 8, 64, 509, 5),
        # a few requests forked at a partly filled page, all 32 layers of an 8B model in one call
        _copy("copy-forks", "bf16", 4, 4, 32, 8, 128),
        # a pool of one layer being compacted: 4096 pages on the move, a list with as many unused places
        _copy("copy-compaction", "bf16", 4096, 4096, 1, 8, 128),
        # the step of a continuous batch: a tenth has finished, as many new prompts, windows that have moved on
        _remap("remap-step", "step", 128, 128, 128, 8192, 7, 0, 1024, 4, 1.3),
        # 16 prompts of 4K tokens with a common beginning become 256 samples
        _remap("remap-fork", "fork", 16, 256, 2048, 4096, 4, 64, 0, 0, 2.0),
        # a small pool after a burst has drained
        _compact("compact-small", 2048, 600, 16),
        # a pool that fills the card's memory, half used
        _compact("compact-pool", 262144, 131000, 512),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (query heads, kv heads, head dim): the configurations' head layouts and those between them
_HEADS = ((32, 32, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (16, 2, 128), (8, 8, 64), (32, 8, 64), (14, 2, 64))
_MOST_KV_BYTES = 8e8          # visible K and V of one pass: below the largest listed case
_MOST_COPY_BYTES = 2.4e8      # bytes of K and V that one pass reads


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(("attn", "attn", "attn", "copy", "remap", "compact"))
    if kind == "attn":
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        hq, hkv, d = rng.choice(_HEADS)
        spec_hi = rng.randint(0, 8)
        spec_lo = rng.randint(0, spec_hi)
        ctx_hi = _log(rng, 24, 65536 if dtype != "f32" else 4096)
        ctx_lo = max(spec_hi + 1, int(ctx_hi * rng.uniform(0.05, 1.0)))
        ctx_hi = max(ctx_hi, ctx_lo)
        window = _log(rng, 1, 4096 if dtype != "f32" else 1024)
        sinks = rng.choice((0, 0, 1, 4, 4, rng.randint(2, 80)))
        seen = min(ctx_hi, window + sinks + spec_hi + 32)
        most = _MOST_KV_BYTES if dtype != "f32" else 4e7
        batch = _log(rng, 1, max(1, min(256 if dtype != "f32" else 16, int(most / (2.0 * hkv * d * _SIZE[dtype] * seen)))))
        return dict(kind=kind, dtype=dtype, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, spec_lo=spec_lo, spec_hi=spec_hi, hq=hq,
                    hkv=hkv, d=d, window=window, sinks=sinks)
    if kind == "copy":
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        _, hkv, d = rng.choice(_HEADS)
        layers = rng.choice((1, 1, 4, rng.randint(2, 40)))
        pairs = _log(rng, 1, max(1, min(8192, int(_MOST_COPY_BYTES / (2.0 * layers * hkv * PAGE * d * _SIZE[dtype])))))
        return dict(kind=kind, dtype=dtype, pairs=pairs, padding=rng.choice((0, rng.randint(1, 2 * pairs))), layers=layers, hkv=hkv,
                    d=d)
    if kind == "remap":
        old_batch, batch = _log(rng, 1, 512), _log(rng, 1, 512)
        ctx_hi = _log(rng, 32, min(65536, (1 << 22) // max(old_batch, batch)))
        window = rng.choice((0, _log(rng, 1, 4096)))
        return dict(kind=kind, mode=rng.choice(("step", "fork")), old_batch=old_batch, batch=batch,
                    ctx_lo=max(2, int(ctx_hi * rng.uniform(0.05, 1.0))), ctx_hi=ctx_hi, grow=rng.randint(1, 40),
                    shared=rng.randint(0, ctx_hi // PAGE), window=window, sinks=rng.choice((0, 4, rng.randint(1, 80))) if window else 0,
                    room=rng.choice((0.8, 1.1, 1.5, 2.0)))
    num_pages = _log(rng, 16, 262144)
    return dict(kind=kind, num_pages=num_pages, used=rng.randint(1, num_pages), batch=_log(rng, 1, 512))


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
class _State:
    pass


def _randn(shape, gen, dtype, sigma=1.0):
    x = torch.empty(shape, dtype=_TORCH[dtype], device="cuda")
    x.normal_(0.0, sigma, generator=gen)
    return x


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _quantiles(lo, hi, n):
    return [lo + int((hi - lo) * (i + 0.5) / n) for i in range(n)]


def _spec_list(c):
    lo, hi, n = c["spec_lo"], c["spec_hi"], c["batch"]
    return [lo + min(hi - lo, int((hi - lo + 1) * (i + 0.5) / n)) for i in range(n)]


def _visible_pages(L, n, window, sinks):
    """Page indices of a request that some of its rows look at."""
    low = max(0, L - n - window + 1) // PAGE
    first = min(-(-sinks // PAGE), low)
    return list(range(first)) + list(range(low, -(-L // PAGE)))


def _prepare_attn(s, c, r, gen):
    spec, ctx = _spec_list(c), _quantiles(c["ctx_lo"], c["ctx_hi"], c["batch"])
    r.shuffle(spec)
    r.shuffle(ctx)
    s.spec_list, s.ctx_list = spec, ctx
    pages = [_visible_pages(L, k + 1, c["window"], c["sinks"]) for L, k in zip(ctx, spec)]
    need = sum(len(p) for p in pages)
    ids = list(range(max(1, math.ceil(1.25 * need))))
    r.shuffle(ids)
    table = torch.full((len(ctx), max(p[-1] for p in pages) + 1), -1, dtype=torch.int32)
    at = 0
    for i, p in enumerate(pages):
        table[i, torch.tensor(p)] = torch.tensor(ids[at:at + len(p)], dtype=torch.int32)
        at += len(p)
    s.block_table, s.ctx_lens, s.spec_lens = table.cuda(), _ints(ctx), _ints(spec)
    kv = (len(ids), c["hkv"], PAGE, c["d"])
    s.k_pages, s.v_pages = _randn(kv, gen, c["dtype"]), _randn(kv, gen, c["dtype"])
    s.q = _randn((sum(spec) + len(spec), c["hq"], c["d"]), gen, c["dtype"])
    if c["sinks"]:
        # what keeps first tokens visible for: every query leans towards their keys
        lean = torch.randn(c["d"], generator=gen, device="cuda").mul_(c["d"] ** -0.25)
        s.q.add_(lean.to(s.q.dtype))
        first = s.block_table[:, 0].long()
        s.k_pages[first, :, : min(PAGE, c["sinks"])] += (2.0 * lean).to(s.q.dtype)


def _prepare_copy(s, c, r, gen):
    pool = 2 * c["pairs"] + c["pairs"] // 4 + 1
    kv = (c["layers"], pool, c["hkv"], PAGE, c["d"])
    s.k_pages, s.v_pages = _randn(kv, gen, c["dtype"]), _randn(kv, gen, c["dtype"])
    ids = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    unused = torch.full((c["padding"],), -1, dtype=torch.int32, device="cuda")
    s.copy_src = torch.cat([ids[:c["pairs"]], unused])
    s.copy_dst = torch.cat([ids[c["pairs"]:2 * c["pairs"]], unused])


def _refs(table, num_pages):
    held = table.long().clamp(min=-1).reshape(-1)
    return torch.zeros(num_pages + 1, dtype=torch.int32, device="cuda").index_add_(
        0, torch.where(held < 0, num_pages, held), torch.ones_like(held, dtype=torch.int32))[:num_pages].contiguous()


def _remap_width(c):
    return -(-(c["ctx_hi"] + c["grow"]) // PAGE)


def _remap_pages(c):
    """Pages of the pool: what the old batch holds and about what the new one wants, times the case's room."""
    held = sum(-(-L // PAGE) for L in _quantiles(c["ctx_lo"], c["ctx_hi"], c["old_batch"]))
    prompts = max(0, c["batch"] - max(1, int(0.9 * c["old_batch"]))) if c["mode"] == "step" else 0
    wanted = c["batch"] * (1 + c["grow"] // PAGE) + prompts * (c["ctx_lo"] + c["ctx_hi"]) // (2 * PAGE)
    return max(held, 1, int(c["room"] * (held + wanted)))


def _prepare_remap(s, c, r, gen):
    old, new, P = c["old_batch"], c["batch"], PAGE
    ctx = _quantiles(c["ctx_lo"], c["ctx_hi"], old)
    r.shuffle(ctx)
    prompts = _quantiles(c["ctx_lo"], c["ctx_hi"], new)
    r.shuffle(prompts)
    # the last step reserved pages for drafts of which some were rejected
    lens = [L - r.randrange(0, min(L, c["grow"])) for L in ctx]
    if c["mode"] == "step":
        stay = r.sample(range(old), min(new, max(1, int(0.9 * old))))
        sources = sorted(stay) + [-1] * (new - len(stay))
    else:
        sources = [r.randrange(old) for _ in range(new)]
    new_lens = [lens[j] + 1 + r.randrange(c["grow"]) if j >= 0 else prompts[i] for i, j in enumerate(sources)]
    width = _remap_width(c)
    held = [-(-L // P) for L in ctx]
    s.num_pages = _remap_pages(c)
    ids = torch.randperm(s.num_pages, generator=gen, device="cuda").to(torch.int32)
    n_held = _ints(held).long()
    base = (n_held.cumsum(0) - n_held)[:, None]
    j = torch.arange(width, device="cuda")
    table = ids[(base + j).clamp(max=s.num_pages - 1)]
    if c["shared"]:         # pairs of rows with a common beginning: whole pages that both hold
        lead = torch.arange(old, device="cuda") // 2 * 2
        common = torch.minimum(n_held, n_held[lead])[:, None] - 1
        table = torch.where(j < common.clamp(max=c["shared"]), table[lead], table)
    table = torch.where(j < n_held[:, None], table, -1)
    s.page_refs = _refs(table, s.num_pages)
    s.block_table = table.to(torch.int32).contiguous()
    s.sources, s.lens, s.new_lens = _ints(sources), _ints(lens), _ints(new_lens)


def _prepare_compact(s, c, r, gen):
    B, used = c["batch"], c["used"]
    ids = torch.randperm(c["num_pages"], generator=gen, device="cuda")[:used].to(torch.int32)
    # rows of every length up to twice the mean
    rows = [used * (i + 1) ** 2 // B ** 2 - used * i ** 2 // B ** 2 for i in range(B)]
    width = max(1, max(rows))
    r.shuffle(rows)
    held = _ints(rows).long()[:, None]
    start = held.cumsum(0) - held
    j = torch.arange(width, device="cuda")
    table = torch.where(j < held, ids[(start + j).clamp(max=used - 1)], -1)
    if B > 1:               # the second row shares the beginning of the first
        both = torch.minimum(held[0], held[1])
        table[1] = torch.where(j < both // 2, table[0], table[1])
    s.block_table = table.to(torch.int32).contiguous()
    s.page_refs = _refs(table, c["num_pages"])


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    {"attn": _prepare_attn, "copy": _prepare_copy, "remap": _prepare_remap, "compact": _prepare_compact}[case["kind"]](
        s, case, random.Random("inputs %d" % seed), gen)
    return s


# --------------------------------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------------------------------
def _plain_attn(s, c):
    W, S, B, hkv, d = c["window"], c["sinks"], c["batch"], c["hkv"], c["d"]
    G, dev, most = c["hq"] // c["hkv"], s.q.device, c["spec_hi"] + 1
    n, L = s.spec_lens.long() + 1, s.ctx_lens.long()
    # the tokens a request looks at: its first S, and from the oldest that its first row's window holds on
    span = min(c["ctx_hi"], W + most - 1)
    low = (L - n - W + 1).clamp(min=0)
    first = torch.arange(min(S, c["ctx_hi"]), device=dev).expand(B, -1)
    last = low[:, None] + torch.arange(span, device=dev)
    t = torch.cat([first, last], dim=1)
    there = torch.cat([first < torch.minimum(low, L)[:, None], last < L[:, None]], dim=1)
    page = s.block_table.long().gather(1, (t // PAGE).clamp(max=s.block_table.shape[1] - 1))
    page = torch.where(there, page, 0)
    k = s.k_pages[page, :, t % PAGE].float().permute(0, 2, 3, 1).contiguous()           # [B][Hkv][d][T]
    v = s.v_pages[page, :, t % PAGE].float().permute(0, 2, 1, 3).contiguous()           # [B][Hkv][T][d]
    # rows padded to the longest request
    start = n.cumsum(0) - n
    j = torch.arange(most, device=dev)
    row = (start[:, None] + torch.minimum(j, n[:, None] - 1))                          # [B][n]
    pos = (L - n)[:, None] + j
    q = s.q[row].float().view(B, most, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, most * G, d)
    score = torch.matmul(q, k) * d ** -0.5
    tt, pp = t[:, None, :], pos[:, :, None]
    sees = there[:, None, :] & (tt <= pp) & ((tt > pp - W) | (tt < S))
    score = score.view(B, hkv, most, G, -1).masked_fill(~sees[:, None, :, None], float("-inf"))
    # (a padding row may see nothing: its maximum is put at 0)
    top = score.amax(dim=-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == float("-inf"), 0.0, top))
    out = torch.matmul(weight.view(B, hkv, most * G, -1), v).view(B, hkv, most, G, d) / weight.sum(dim=-1, keepdim=True)
    out = out.permute(0, 2, 1, 3, 4).reshape(B * most, c["hq"], d)
    real = torch.arange(s.q.shape[0], device=dev)
    owner = torch.searchsorted(n.cumsum(0), real, right=True)
    return out[owner * most + real - start[owner]].to(s.q.dtype)


def _plain_copy(s, c):
    there = s.copy_src >= 0
    src, dst = s.copy_src[there].long(), s.copy_dst[there].long()
    s.k_pages[:, dst] = s.k_pages[:, src]
    s.v_pages[:, dst] = s.v_pages[:, src]
    return {"k_pages": s.k_pages, "v_pages": s.v_pages}


def _held(refs, pages, by):
    """refs + by for every page in `pages` that is one (the entry behind the last page takes the others)"""
    NP = refs.shape[0]
    pages = pages.reshape(-1).long()
    more = torch.cat([refs, refs.new_zeros(1)])
    return more.index_add_(0, torch.where((pages >= 0) & (pages < NP), pages, NP), torch.full_like(pages, by, dtype=refs.dtype))[:NP]


def _plain_remap(s, c):
    table, refs, NP = s.block_table, s.page_refs, s.num_pages
    B, dev, width = s.sources.shape[0], s.sources.device, s.block_table.shape[1]
    src = s.sources.long()
    old = src >= 0
    lens = torch.where(old, s.lens.long()[src.clamp(min=0)], 0)
    j = torch.arange(width, device=dev)
    kept = j < ((lens + PAGE - 1) // PAGE)[:, None]
    if c["window"]:
        behind = ((lens - c["window"] + 1).clamp(min=0) // PAGE)[:, None]
        kept = kept & ((j >= behind) | (j < -(-c["sinks"] // PAGE)))
    out = torch.where(kept & old[:, None], table[src.clamp(min=0)], -1)
    refs = _held(_held(refs, table, -1), out, 1)
    # whoever writes into a page that others hold as well wants a copy; of those who share it the last keeps it
    part = torch.where((lens % PAGE != 0) & (s.new_lens > lens), out.gather(1, (lens // PAGE).clamp(max=width - 1)[:, None])[:, 0], -1)
    before = ((part[:, None] == part[None, :]).tril(-1)).sum(dim=1)
    copies = (part >= 0) & (before < refs[part.clamp(min=0).long()] - 1)
    begin = (lens + PAGE - 1) // PAGE
    end = ((s.new_lens.long() + PAGE - 1) // PAGE).clamp(max=width)
    wants = copies.long() + (end - begin).clamp(min=0)
    base = wants.cumsum(0) - wants
    # free pages in ascending order
    free = refs == 0
    ranks = torch.where(free, free.cumsum(0) - 1, NP)
    pages = torch.full((NP + 1,), -1, dtype=torch.int32, device=dev)
    pages[ranks] = torch.arange(NP, dtype=torch.int32, device=dev)
    n_free, total = free.sum(), wants.sum()
    pages = torch.where(torch.arange(NP + 1, device=dev) < n_free, pages, -1)
    fresh = (j >= begin[:, None]) & (j < end[:, None])
    got = pages[(base[:, None] + copies[:, None] + j - begin[:, None]).clamp(min=0, max=NP)]
    out = torch.where(fresh, got, out)
    private = torch.where(copies, pages[base.clamp(max=NP)], -1)
    served = private >= 0
    out = torch.where((j == (lens // PAGE)[:, None]) & served[:, None], private[:, None], out)
    copy_src = torch.where(served, part, -1)
    refs = _held(_held(_held(refs, torch.where(fresh, got, -1), 1), private, 1), copy_src, -1)
    status = torch.stack([n_free - torch.minimum(n_free, total), (total - n_free).clamp(min=0)]).to(torch.int32)
    return {"table": out, "refs": refs, "copy_src": copy_src, "copy_dst": private, "status": status}


def _plain_compact(s, c):
    refs, NP = s.page_refs, c["num_pages"]
    dev, most = refs.device, max(1, c["num_pages"] // 2)
    page = torch.arange(NP, device=dev)
    used = refs > 0
    N = used.sum()
    holes, movers = ~used & (page < N), used & (page >= N)
    lists = torch.full((2, most + 1), -1, dtype=torch.int32, device=dev)
    lists[0, torch.where(movers, movers.cumsum(0) - 1, most)] = page.to(torch.int32)
    lists[1, torch.where(holes, holes.cumsum(0) - 1, most)] = page.to(torch.int32)
    moves = movers.sum()
    lists = torch.where(torch.arange(most + 1, device=dev) < moves, lists, -1)
    copy_src, copy_dst = lists[0, :most], lists[1, :most]
    to = torch.where(movers, lists[1][(movers.cumsum(0) - 1).clamp(min=0)], page.to(torch.int32))
    page_map = torch.where(used, to, -1)
    new_refs = torch.zeros(NP + 1, dtype=torch.int32, device=dev)
    new_refs[torch.where(used, page_map, NP).long()] = refs
    table = torch.where(s.block_table >= 0, page_map[s.block_table.clamp(min=0).long()], -1)
    status = torch.stack([N, moves]).to(torch.int32)
    return {"table": table, "refs": new_refs[:NP], "map": page_map, "copy_src": copy_src, "copy_dst": copy_dst, "status": status}


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------
def _own(s, c):
    import paper_2503_05096_amd as pkg
    if c["kind"] == "attn":
        return {"out": pkg.verify_attn(s.q, s.k_pages, s.v_pages, s.block_table, s.ctx_lens, s.spec_lens, max_spec_len=c["spec_hi"],
                                       window=c["window"], sinks=c["sinks"])}
    if c["kind"] == "copy":
        pkg.kv_copy_pages(s.k_pages, s.v_pages, s.copy_src, s.copy_dst)
        return {"k_pages": s.k_pages, "v_pages": s.v_pages}
    if c["kind"] == "remap":
        table, refs, copy_src, copy_dst, status = pkg.kv_remap(s.block_table, s.page_refs, s.sources, s.lens, s.new_lens,
                                                               window=c["window"] or None, sinks=c["sinks"])
        return {"table": table, "refs": refs, "copy_src": copy_src, "copy_dst": copy_dst, "status": status}
    table, refs, page_map, copy_src, copy_dst, status = pkg.kv_compact_pages(s.block_table, s.page_refs)
    return {"table": table, "refs": refs, "map": page_map, "copy_src": copy_src, "copy_dst": copy_dst, "status": status}


def run(s):
    c = s.case
    if own:
        return _own(s, c)
    if c["kind"] == "attn":
        return {"out": _plain_attn(s, c)}
    return {"copy": _plain_copy, "remap": _plain_remap, "compact": _plain_compact}[c["kind"]](s, c)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------
def _work_attn(c):
    spec, ctx = _spec_list(c), _quantiles(c["ctx_lo"], c["ctx_hi"], c["batch"])
    # (which length meets which draft length is the seed's choice: the mean draft length stands for all)
    n_mean = sum(spec) / len(spec) + 1.0
    W, S, size = c["window"], c["sinks"], _SIZE[c["dtype"]]
    tokens = seen = 0.0
    for L in ctx:
        low = max(0.0, L - n_mean - W + 1)
        tokens += (L - low) + min(S, low)
        seen += min(L - (n_mean - 1) / 2, W + min(S, max(0.0, L - W)))
    rows = sum(spec) + len(spec)
    kv = tokens * 2 * c["hkv"] * c["d"] * size
    table = tokens / PAGE * 4
    return {"bytes": int(kv + table + 2 * rows * c["hq"] * c["d"] * size + 8 * len(ctx)),
            "flops": int(4 * c["d"] * c["hq"] * n_mean * seen)}


def work(c):
    if c["kind"] == "attn":
        return _work_attn(c)
    if c["kind"] == "copy":
        page = 2 * c["layers"] * c["hkv"] * PAGE * c["d"] * _SIZE[c["dtype"]]
        return {"bytes": 2 * c["pairs"] * page + 8 * (c["pairs"] + c["padding"]), "flops": 0}
    if c["kind"] == "remap":
        ctx = _quantiles(c["ctx_lo"], c["ctx_hi"], c["old_batch"])
        held = sum(-(-L // PAGE) for L in ctx)
        return {"bytes": 4 * held + 4 * c["batch"] * _remap_width(c) + 8 * _remap_pages(c) + 4 * (5 * c["batch"] + c["old_batch"]),
                "flops": 0}
    return {"bytes": 4 * (2 * c["used"] + 4 * c["num_pages"]), "flops": 0}


# --------------------------------------------------------------------------------------------------
# from the definitions, in 64 bits
# --------------------------------------------------------------------------------------------------
def _exact_attn(s, c):
    W, S, G, d = c["window"], c["sinks"], c["hq"] // c["hkv"], c["d"]
    out = torch.empty(s.q.shape, dtype=torch.float64, device=s.q.device)
    table, at = s.block_table.cpu(), 0
    for i, (L, k) in enumerate(zip(s.ctx_list, s.spec_list)):
        first_row = L - k - 1
        tokens = [t for t in range(min(S, L))] + list(range(max(S, first_row - W + 1, 0), L))
        t = torch.tensor(tokens)
        page, slot = table[i, t // PAGE].long().to(out.device), (t % PAGE).to(out.device)
        keys, values = s.k_pages[page, :, slot].double(), s.v_pages[page, :, slot].double()     # [T][Hkv][d]
        t = t.to(out.device)
        for j in range(k + 1):
            sees = (t <= first_row + j) & ((first_row + j - t < W) | (t < S))
            q = s.q[at + j].double().view(c["hkv"], G, d)
            score = (q[:, :, None, :] * keys[sees].transpose(0, 1)[:, None]).sum(-1) / math.sqrt(d)      # [Hkv][G][T]
            p = torch.exp(score - torch.logsumexp(score, dim=-1, keepdim=True))
            out[at + j] = (p[..., None] * values[sees].transpose(0, 1)[:, None]).sum(2).reshape(c["hq"], d)
        at += k + 1
    return {"out": out}


def _exact_remap(s, c):
    table, refs = s.block_table.tolist(), s.page_refs.tolist()
    sources, lens, new_lens = s.sources.tolist(), s.lens.tolist(), s.new_lens.tolist()
    width = s.block_table.shape[1]
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    out, keep = [], []
    for j in sources:
        n = lens[j] if j >= 0 else 0
        row = [-1] * width
        for x in range(-(-n // PAGE)):
            hidden = c["window"] > 0 and PAGE * x >= c["sinks"] and PAGE * x + PAGE - 1 <= n - c["window"]
            if not hidden:
                row[x] = table[j][x]
                if row[x] >= 0:
                    refs[row[x]] += 1
        out.append(row)
        keep.append(n)
    free = [p for p, r in enumerate(refs) if r == 0]
    shared, wants = list(refs), []
    for i, row in enumerate(out):
        n, end = keep[i], min(width, -(-new_lens[i] // PAGE))
        if n % PAGE and new_lens[i] > n:
            p = row[n // PAGE]
            if p >= 0 and shared[p] > 1:
                shared[p] -= 1
                wants.append((i, n // PAGE, p))
        wants += [(i, x, -1) for x in range(-(-n // PAGE), end)]
    copy_src, copy_dst = [-1] * len(out), [-1] * len(out)
    for (i, x, p), f in zip(wants, free):
        out[i][x] = f
        refs[f] += 1
        if p >= 0:
            copy_src[i], copy_dst[i] = p, f
            refs[p] -= 1
    status = [max(0, len(free) - len(wants)), max(0, len(wants) - len(free))]
    as_ints = lambda v: torch.tensor(v, dtype=torch.int32)                                     # noqa: E731
    return {"table": as_ints(out), "refs": as_ints(refs), "copy_src": as_ints(copy_src), "copy_dst": as_ints(copy_dst),
            "status": as_ints(status)}


def _exact_compact(s, c):
    table, refs = s.block_table.tolist(), s.page_refs.tolist()
    used = [p for p, r in enumerate(refs) if r > 0]
    N, taken = len(used), set(used)
    movers, holes = [p for p in used if p >= N], [p for p in range(N) if p not in taken]
    to = {p: p for p in used}
    to.update(zip(movers, holes))
    new_refs = [0] * len(refs)
    for p in used:
        new_refs[to[p]] = refs[p]
    unused = [-1] * (max(1, len(refs) // 2) - len(movers))
    as_ints = lambda v: torch.tensor(v, dtype=torch.int32)                                     # noqa: E731
    return {"table": as_ints([[to[p] if p >= 0 else -1 for p in row] for row in table]), "refs": as_ints(new_refs),
            "map": as_ints([to.get(p, -1) for p in range(len(refs))]), "copy_src": as_ints(movers + unused),
            "copy_dst": as_ints(holes + unused), "status": as_ints([N, len(movers)])}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(s, case)
    if case["kind"] == "remap":
        return _exact_remap(s, case)
    if case["kind"] == "compact":
        return _exact_compact(s, case)
    k, v = s.k_pages.double(), s.v_pages.double()
    for a, b in zip(s.copy_src.tolist(), s.copy_dst.tolist()):
        if a >= 0:
            k[:, b] = k[:, a]
            v[:, b] = v[:, a]
    return {"k_pages": k, "v_pages": v}
