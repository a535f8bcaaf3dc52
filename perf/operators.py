"""The operators of long-context serving around the fused attention, as cases to be timed: attention with a
sliding window and a few first tokens that stay visible, a cache of keys and values in 8 bits (E4M3 codes with a
power-of-two scale per page and head), the attention of new tokens over that cache, and the management of its pages.

A case is a dict of plain values; ``op`` names the operator:
  window    prompt prefill: key c is visible to query r where c <= r and (c > r - window or c < sinks)
  append    new keys and values into the pages of the cache: scales, codes, old codes of a page whose scale grows
  cache     attention of the last T tokens of each sequence over the cache
  fork      the rows of a batch rebuilt from parents: full pages shared, last pages copied, pages reserved
  compact   the pages in use moved to the front of the pool
Shapes of heads are those of the prefill and encoder workloads of this repository (32 query heads on 8 or 32 kv heads
of 128, 16 heads of 64).
"""
import math

import torch

own = False
LOG2E = 1.4426950408889634
NO_WINDOW = 2 ** 31 - 1
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # a short prompt of odd length on few heads: all latency
        {"name": "window_short_prompt", "op": "window", "B": 1, "H": 4, "Hkv": 2, "S": 333, "D": 128, "window": 128,
         "sinks": 4, "type": "bf16", "ragged": False},
        # a padded batch of prompts, heads of 64, a narrow window
        {"name": "window_ragged_d64", "op": "window", "B": 8, "H": 16, "Hkv": 4, "S": 4001, "D": 64, "window": 500,
         "sinks": 20, "type": "f16", "ragged": True},
        # one long prompt, grouped kv heads
        {"name": "window_long_prompt", "op": "window", "B": 1, "H": 32, "Hkv": 8, "S": 32768, "D": 128, "window": 4096,
         "sinks": 64, "type": "bf16", "ragged": False},
        # one new token for each sequence of a decoding batch
        {"name": "append_one_token", "op": "append", "B": 96, "Hkv": 8, "D": 128, "page": 64, "new": 1, "held": 4000,
         "type": "bf16"},
        # prompts of different lengths that arrive together, some behind a shared prefix
        {"name": "append_prompts", "op": "append", "B": 12, "Hkv": 8, "D": 128, "page": 64, "new": 8192, "held": 700,
         "type": "bf16"},
        # one request, one token: latency
        {"name": "cache_one_request", "op": "cache", "B": 1, "H": 32, "Hkv": 8, "T": 1, "D": 128, "page": 64,
         "context": 2000, "window": NO_WINDOW, "sinks": 0, "type": "bf16"},
        # drafts of four tokens being verified, windowed, heads of 64, small pages
        {"name": "cache_drafts_window", "op": "cache", "B": 32, "H": 16, "Hkv": 4, "T": 4, "D": 64, "page": 16,
         "context": 16000, "window": 4096, "sinks": 4, "type": "f16"},
        # a decoding batch of long contexts of different lengths
        {"name": "cache_long_batch", "op": "cache", "B": 48, "H": 32, "Hkv": 8, "T": 1, "D": 128, "page": 64,
         "context": 32768, "window": NO_WINDOW, "sinks": 0, "type": "bf16"},
        # four beams of one request
        {"name": "fork_beams", "op": "fork", "rows": 4, "new_rows": 4, "Hkv": 8, "D": 128, "page": 64, "context": 1500,
         "reserve": 1, "window": NO_WINDOW, "sinks": 0},
        # a serving batch rebuilt: some requests sampled several times, some gone, old pages released
        {"name": "fork_batch_window", "op": "fork", "rows": 128, "new_rows": 256, "Hkv": 8, "D": 128, "page": 32,
         "context": 9000, "reserve": 4, "window": 4096, "sinks": 4},
        # a small pool with a few holes
        {"name": "compact_small_pool", "op": "compact", "rows": 6, "pages": 300, "Hkv": 4, "D": 64, "page": 16, "live": 0.7},
        # a pool half of which is free after many requests have ended
        {"name": "compact_half_free", "op": "compact", "rows": 64, "pages": 9001, "Hkv": 8, "D": 128, "page": 64, "live": 0.5},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["window", "window", "append", "cache", "cache", "fork", "compact"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    kind = rng.choice(["bf16", "bf16", "f16"])
    page = rng.choice([16, 32, 64, 128])
    case = {"op": op, "Hkv": Hkv, "D": D}
    if op == "window":
        while True:
            H = Hkv * rng.choice([1, 2, 3, 4, 8])
            B, S = _log_uniform(rng, 1, 16), _log_uniform(rng, 1, 32768)
            window = _log_uniform(rng, 1, 8192)
            # (no more scores, and no more memory in the plain form, than the largest listed case)
            if H <= 32 and B * H * S * (min(window, S) + 1024) <= 32 * 32768 * 5000 and B * H * S * D <= 32 * 32768 * 128:
                break
        return {**case, "B": B, "H": H, "S": S, "window": window, "sinks": rng.choice([0, 1, 4, 37, 128]), "type": kind,
                "ragged": rng.random() < 0.4}
    if op == "append":
        new = rng.choice([1, 1, 2, 5, _log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 8192)])
        B = min(_log_uniform(rng, 1, 200), max(1, 90000 // new))
        return {**case, "B": B, "page": page, "new": new, "held": _log_uniform(rng, 1, 5000), "type": kind}
    if op == "cache":
        T = rng.choice([1, 1, 1, 2, 3, 5, 8])
        context = _log_uniform(rng, 1, 131072)
        B = min(_log_uniform(rng, 1, 128), max(1, 48 * 32768 * 1024 // (context * Hkv * D)))
        H = Hkv * rng.choice([1, 2, 3, 4, 8])
        if rng.random() < 0.5:
            window, sinks = NO_WINDOW, 0
        else:
            window, sinks = _log_uniform(rng, 16, 8192), rng.choice([0, 1, 4, 100])
        return {**case, "B": B, "H": H, "T": T, "page": page, "context": context, "window": window, "sinks": sinks, "type": kind}
    if op == "fork":
        rows = _log_uniform(rng, 1, 128)
        context = min(_log_uniform(rng, 1, 20000), 1200000 // rows)
        windowed = rng.random() < 0.5
        return {**case, "rows": rows, "new_rows": rng.randint(1, 2 * rows), "page": page, "context": context,
                "reserve": rng.choice([0, 1, 4, 200]), "window": _log_uniform(rng, 16, 8192) if windowed else NO_WINDOW,
                "sinks": rng.choice([0, 4, 100]) if windowed else 0}
    pages = _log_uniform(rng, 10, 9000 * 65536 // (Hkv * page * D) if Hkv * page * D > 65536 else 9000)
    return {**case, "rows": _log_uniform(rng, 1, 128), "pages": pages, "page": page, "live": rng.choice([0.2, 0.5, 0.8, 0.97])}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rand_int(g, lo, hi, n):
    """n whole numbers in [lo, hi], int32."""
    return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)


def _pool(case, n_pages, g):
    """Pages that hold codes of unit-Gaussian values with scales around 2^-7: what earlier tokens left there."""
    shape = (n_pages, case["Hkv"], case["page"], case["D"])
    pool = {}
    for n in ("k", "v"):
        codes = torch.empty(shape, device="cuda", dtype=torch.uint8)
        flat = codes.view(-1)
        for part in flat.split(1 << 28):                      # (in pieces: a float32 copy of the pool need not fit)
            part.copy_((torch.randn(part.numel(), generator=g, device="cuda") * 100).clamp_(-448, 448)
                       .to(torch.float8_e4m3fn).view(torch.uint8))
        pool[n] = codes
        e = torch.randint(-8, -5, shape[:2], generator=g, device="cuda").float()
        pool[n + "_scale"] = torch.exp2(e)
    return pool


def _table(held_pages, width, n_pages, g, refs=None):
    """Rows of pages in random order, no page in two rows; -1 behind a row's last page."""
    rows = held_pages.numel()
    order = torch.randperm(n_pages, generator=g, device="cuda")[:rows * width].to(torch.int32).view(rows, width)
    col = torch.arange(width, device="cuda")
    return torch.where(col < held_pages[:, None], order, -1).to(torch.int32).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    state = {"case": case}
    if op == "window":
        B, H, Hkv, S, D = (case[n] for n in ("B", "H", "Hkv", "S", "D"))
        dt = TYPES[case["type"]]
        # the projections' layout: [B, S, heads, D], seen as [B, heads, S, D]
        for n, h in (("q", H), ("k", Hkv), ("v", Hkv)):
            state[n] = torch.randn(B, S, h, D, generator=g, device="cuda").to(dt).transpose(1, 2)
        state["lengths"] = _rand_int(g, max(1, S // 4), S, B) if case["ragged"] else None
        state["out"] = torch.zeros(B, S, H, D, device="cuda", dtype=dt).transpose(1, 2)
        state["lse"] = torch.zeros(B, H, S, device="cuda")
        return state
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    if op == "append":
        B, new, dt = case["B"], case["new"], TYPES[case["type"]]
        counts = torch.full((B,), new, device="cuda", dtype=torch.int32) if new <= 5 else _rand_int(g, max(1, new // 3), new, B)
        held = _rand_int(g, 0, 2 * case["held"], B)
        held[::3] = 0                                        # some sequences begin here
        starts = torch.zeros(B + 1, device="cuda", dtype=torch.int32)
        starts[1:] = counts.cumsum(0)
        width = (2 * case["held"] + new) // page + 1
        # (pages that no token of this call goes to are left out of the pool: the table names only those it needs)
        first, last = held // page, (held + counts - 1) // page
        col = torch.arange(width, device="cuda")
        here = (col >= first[:, None]) & (col <= last[:, None])
        used = here.flatten().long().cumsum(0).view(B, width)
        n_pages = B * ((new + page - 1) // page + 1)
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        state["table"] = torch.where(here, order[(used - 1).clamp(0)], -1).to(torch.int32).contiguous()
        state.update(_pool(case, n_pages, g), lengths=held, starts=starts, max_new=new)
        n = int(starts[-1])
        # keys and values behind the queries of one projection; a few tokens are much larger than the rest
        qkv = torch.randn(n, 3 * Hkv, D, generator=g, device="cuda")
        qkv *= torch.where(torch.rand(n, 1, 1, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        qkv = qkv.to(dt)
        state["k_new"], state["v_new"] = qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:]
        return state
    if op == "cache":
        B, H, T, dt = case["B"], case["H"], case["T"], TYPES[case["type"]]
        context = case["context"]
        lengths = _rand_int(g, max(1, context // 4), context, B)
        lengths[0] = context
        width = (context + page - 1) // page
        held = (lengths + page - 1) // page
        # pages that left the window have been given back
        first_query = lengths - T
        col = torch.arange(width, device="cuda")
        seen = (col * page < case["sinks"]) | ((col + 1) * page - 1 > (first_query.long() - case["window"])[:, None])
        here = seen & (col < held[:, None])
        used = here.flatten().long().cumsum(0).view(B, width)
        n_pages = max(1, int(here.sum()))
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        state["table"] = torch.where(here, order[(used - 1).clamp(0)], -1).to(torch.int32).contiguous()
        state.update(_pool(case, n_pages, g), lengths=lengths)
        state["q"] = torch.randn(B, T, H, D, generator=g, device="cuda").to(dt).transpose(1, 2)
        return state
    if op == "fork":
        rows, new_rows, context = case["rows"], case["new_rows"], case["context"]
        lengths = _rand_int(g, max(1, context // 4), context, rows)
        held = (lengths + page - 1) // page
        width = (context + case["reserve"] + page - 1) // page
        extra = (case["reserve"] + page - 1) // page + 2
        n_pages = rows * width + new_rows * extra
        state["table"] = _table(held, width, n_pages, g)
        state.update(_pool(case, n_pages, g), lengths=lengths)
        refs = torch.zeros(n_pages + 1, device="cuda", dtype=torch.int32)
        flat = state["table"].flatten().long()
        refs.index_add_(0, torch.where(flat >= 0, flat, n_pages), torch.ones_like(flat, dtype=torch.int32))
        state["refs"] = refs[:n_pages].contiguous()
        parents = _rand_int(g, 0, rows - 1, new_rows)
        parents[new_rows // 2::7] = -1                       # empty places of the batch
        state["parents"] = parents
        return state
    rows, n_pages = case["rows"], case["pages"]
    live = max(1, int(n_pages * case["live"]))
    width = (live + rows - 1) // rows
    held = torch.full((rows,), width, device="cuda", dtype=torch.int32)
    held[-1] = live - (rows - 1) * width if live > (rows - 1) * width else 0
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(rows * width, device="cuda")
    state["table"] = torch.where(at < live, order[at.clamp(max=n_pages - 1)], -1).to(torch.int32).view(rows, width).contiguous()
    state.update(_pool(case, n_pages, g))
    refs = torch.zeros(n_pages, device="cuda", dtype=torch.int32)
    refs[order[:live].long()] = 1
    shared = state["table"][0, :max(1, width // 4)].clone()   # the first row's first pages are a prefix of the second's too
    if rows > 1:
        gone = state["table"][1, :shared.numel()]
        both = (shared >= 0) & (gone >= 0)
        refs[gone[both].long()] -= 1
        refs[shared[both].long()] += 1
        state["table"][1, :shared.numel()] = torch.where(both, shared, gone)
    state["refs"] = refs
    return state


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _softmax_rows(s, mask):
    """Weights, their sum and the maximum of rows of scores, in the scores' type; rows without a visible key give 0."""
    s = s.masked_fill(~mask, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    return p, p.sum(-1, keepdim=True), m


def _plain_window(s):
    case = s["case"]
    q, k, v = (s[n].float() for n in ("q", "k", "v"))
    B, H, S, D = q.shape
    Hkv, sinks = k.shape[1], min(case["sinks"], S)
    W = min(case["window"], S)
    blk = min(S, max(128, min(1024, W)))
    nb = -(-S // blk)
    pad = nb * blk - S
    span = blk + W - 1

    def blocks(x):                                           # [B, Hkv, 1, nb, span, D]: keys of a block of queries
        x = torch.nn.functional.pad(x, (0, 0, W - 1, pad))
        return x.unfold(2, span, blk).transpose(-1, -2)[:, :, None]

    qb = torch.nn.functional.pad(q, (0, 0, 0, pad)).view(B, Hkv, H // Hkv, nb, blk, D) * (1 / math.sqrt(D))
    row = torch.arange(nb * blk, device=q.device).view(nb, blk, 1)
    col = torch.arange(nb, device=q.device).view(nb, 1, 1) * blk + torch.arange(span, device=q.device) - (W - 1)
    near = (col >= 0) & (col <= row) & (col > row - W)
    first = torch.arange(sinks, device=q.device)
    far = (first <= row - W).expand(nb, blk, sinks)          # first tokens that the window has left behind
    score = torch.cat([qb @ blocks(k).transpose(-1, -2), qb @ k[:, :, None, None, :sinks].transpose(-1, -2)], -1)
    p, l, m = _softmax_rows(score, torch.cat([near, far], -1))
    del score
    o = (p[..., :span] @ blocks(v) + p[..., span:] @ v[:, :, None, None, :sinks]) / l
    out = o.view(B, H, nb * blk, D)[:, :, :S].to(s["q"].dtype)
    lse = (m + torch.log(l)).view(B, H, nb * blk)[:, :, :S]
    if s["lengths"] is not None:                             # rows behind a sequence's end stay as they were
        there = (torch.arange(S, device=q.device) < s["lengths"][:, None])[:, None]
        out, lse = torch.where(there[..., None], out, s["out"]), torch.where(there, lse, s["lse"])
    return out, lse


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _plain_append_one(codes, scale, new, page_of, slot, first_page, seq_held):
    x = new.float()
    amax = x.abs().amax(-1)                                  # [N, Hkv]
    need = torch.zeros_like(scale)
    need.scatter_reduce_(0, page_of[:, None].expand_as(amax), amax, "amax", include_self=True)
    # smallest power of two with amax <= 448 * scale
    mant, exp = torch.frexp(need.clamp(min=2.0 ** -100))
    need = torch.ldexp(torch.ones_like(mant), exp - 9 + (mant > 0.875).int())
    kept = seq_held % codes.shape[2] != 0                    # the first page of a sequence holds older tokens
    old = scale[first_page]
    fresh = torch.full_like(scale, 0.0)
    fresh[first_page] = torch.where(kept[:, None], old, 0.0)
    touched = torch.zeros(scale.shape[0], 1, dtype=torch.bool, device=scale.device)
    touched[page_of] = True
    scale.copy_(torch.where(touched, torch.maximum(need, fresh), scale))
    factor = torch.where(kept[:, None], old / scale[first_page], 1.0)
    moved = _e4m3(codes[first_page].view(torch.float8_e4m3fn).float() * factor[:, :, None, None])
    codes[first_page] = moved.view(torch.uint8)
    codes[page_of, :, slot] = _e4m3(x / scale[page_of][..., None]).view(torch.uint8)


def _plain_append(s):
    page = s["case"]["page"]
    n = s["k_new"].shape[0]
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], t, right=True) - 1
    pos = (s["lengths"][seq] + t - s["starts"][seq]).long()
    page_of = s["table"][seq, pos // page].long()
    first_page = s["table"].gather(1, (s["lengths"] // page).long()[:, None])[:, 0].long()
    for n in ("k", "v"):
        _plain_append_one(s[n], s[n + "_scale"], s[n + "_new"], page_of, pos % page, first_page, s["lengths"])
    return [s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["k_scale"], s["v_scale"]]


def _plain_cache(s):
    case = s["case"]
    q = s["q"].float()
    B, H, T, D = q.shape
    Hkv, page = case["Hkv"], case["page"]
    table = s["table"].clamp(0).long()
    n = table.shape[1] * page
    pos = torch.arange(n, device=q.device)
    at = (s["lengths"][:, None] - T + torch.arange(T, device=q.device))[..., None]           # [B, T, 1]
    mask = (pos <= at) & ((pos > at.long() - case["window"]) | (pos < case["sinks"]))        # [B, T, n]

    def values(name):                                        # [B, Hkv, 1, n, D]
        x = s[name].view(torch.float8_e4m3fn)[table].float() * s[name + "_scale"][table][..., None, None]
        x = x.transpose(1, 2).reshape(B, Hkv, 1, n, D)
        return x.masked_fill(~mask.any(1)[:, None, None, :, None], 0.0)

    score = (q * (1 / math.sqrt(D))).view(B, Hkv, H // Hkv, T, D) @ values("k").transpose(-1, -2)
    p, l, m = _softmax_rows(score, mask[:, None, None])
    o = (p @ values("v")) / torch.where(l == 0, 1.0, l)
    return o.view(B, H, T, D).to(s["q"].dtype), (m + torch.log(l)).view(B, H, T)


def _plain_fork(s):
    case = s["case"]
    page, reserve = case["page"], case["reserve"]
    table, lengths, refs, parents = s["table"].long(), s["lengths"].long(), s["refs"], s["parents"].long()
    rows, width = table.shape
    M = parents.numel()
    valid = (parents >= 0) & (parents < rows)
    parent = parents.clamp(0, rows - 1)
    L = torch.where(valid, lengths[parent].clamp(0), 0)
    held, total = (L + page - 1) // page, (L + reserve + page - 1) // page
    fits = valid & (total <= width)
    col = torch.arange(width, device="cuda")
    alive = (col < held[:, None]) & ((col * page < case["sinks"]) | ((col + 1) * page > (L - case["window"] + 1)[:, None]))
    rows_of = torch.where(alive, table[parent], -1)
    index = torch.arange(M, device="cuda")
    oldest = torch.full((rows,), M, device="cuda").scatter_reduce_(0, torch.where(valid, parent, 0), torch.where(valid, index, M), "amin")
    last = rows_of.gather(1, (held - 1).clamp(0, width - 1)[:, None])[:, 0]
    copy = fits & (L % page != 0) & (oldest[parent] != index) & (last >= 0)
    need = torch.where(fits, copy + total - held, 0)
    begin = need.cumsum(0) - need
    rank = (refs == 0).long().cumsum(0)
    ok = fits & (begin + need <= rank[-1])
    # the r-th lowest free page, for every r that can be asked for
    most = M * (reserve // page + 2)
    free = torch.zeros(most + 1, device="cuda", dtype=torch.long)
    free.scatter_(0, torch.where((refs == 0) & (rank <= most), rank - 1, most), torch.arange(refs.numel(), device="cuda"))
    copy = copy & ok
    fresh_at = begin[:, None] + copy[:, None] + col - held[:, None]
    new = torch.where((col >= held[:, None]) & (col < total[:, None]), free[fresh_at.clamp(0, most)], rows_of)
    target = free[begin.clamp(0, most)]
    new = torch.where(copy[:, None] & (col == (held - 1)[:, None]), target[:, None], new)
    new = torch.where(ok[:, None], new, -1)
    new_refs = torch.zeros(refs.numel() + 1, device="cuda", dtype=torch.int32)
    flat = new.flatten()
    new_refs.index_add_(0, torch.where(flat >= 0, flat, refs.numel()), torch.ones_like(flat, dtype=torch.int32))
    src, dst = last[copy], target[copy]
    for n in ("k", "v", "k_scale", "v_scale"):
        s[n][dst] = s[n][src]
    new_lengths = torch.where(valid, torch.where(ok, L, -1), 0)
    return [new.int(), new_lengths.int(), new_refs[:-1], *(s[n].view(torch.float8_e4m3fn) for n in ("k", "v")), s["k_scale"], s["v_scale"]]


def _plain_compact(s):
    table, refs = s["table"].long(), s["refs"]
    n = refs.numel()
    live = refs > 0
    n_live = live.sum()
    index = torch.arange(n, device="cuda")
    src = index[live & (index >= n_live)]                    # in order: the k-th goes to the k-th hole
    dst = index[~live & (index < n_live)]
    page_map = torch.where(live, index, -1)
    page_map[src] = dst
    new_refs = torch.where(index < n_live, refs, 0)
    new_refs[dst] = refs[src]
    for name in ("k", "v", "k_scale", "v_scale"):
        s[name][dst] = s[name][src]
    new_table = torch.where(table >= 0, page_map[table.clamp(0)], -1)
    return [new_table.int(), new_refs.int(), page_map.int(), n_live.int().view(1),
            *(s[name].view(torch.float8_e4m3fn) for name in ("k", "v")), s["k_scale"], s["v_scale"]]


PLAIN = {"window": _plain_window, "append": _plain_append, "cache": _plain_cache, "fork": _plain_fork, "compact": _plain_compact}


# ---- the library's calls --------------------------------------------------------------------------------------------

def _cache_of(binding, s):
    return binding.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])


def _codes(s):
    return [s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn), s["k_scale"], s["v_scale"]]


def _own(s):
    from paper_2602_02071_b200 import binding
    case = s["case"]
    op = case["op"]
    if op == "window":
        binding.baps_attention_window_fwd(s["q"], s["k"], s["v"], window=case["window"], sinks=case["sinks"],
                                          lengths=s["lengths"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    cache = _cache_of(binding, s)
    if op == "append":
        binding.baps_kv_append(cache, s["k_new"], s["v_new"], s["table"], s["lengths"], s["starts"], max_new=s["max_new"])
        return _codes(s)
    if op == "cache":
        return binding.baps_kv_attention(s["q"], cache, s["table"], s["lengths"], window=case["window"],
                                         sinks=case["sinks"], want_lse=True)
    if op == "fork":
        return [*binding.baps_kv_fork(cache, s["table"], s["lengths"], s["refs"], s["parents"], reserve=case["reserve"],
                                      window=case["window"], sinks=case["sinks"]), *_codes(s)]
    return [*binding.baps_kv_compact(cache, s["table"], s["refs"]), *_codes(s)]


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def _visible(rows, window, sinks):
    """Sum over queries 0 .. rows - 1 of the keys that each sees."""
    window, sinks = min(window, rows), min(sinks, rows)
    near = window * (window + 1) // 2 + (rows - window) * window
    far = sum(min(sinks, r - window + 1) for r in range(window, min(rows, window + sinks)))
    far += sinks * max(0, rows - window - sinks)
    return near + far


def work(case):
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    if op == "window":
        B, H, S = case["B"], case["H"], case["S"]
        share = 0.625 if case["ragged"] else 1.0             # the mean length of a ragged batch
        rows = max(1, int(S * share))
        return {"bytes": B * rows * (2 * H + 2 * Hkv) * D * 2 + 4 * B * H * rows,
                "flops": 4 * B * H * D * _visible(rows, case["window"], case["sinks"])}
    page_bytes = 2 * Hkv * (case["page"] * D + 4)
    if op == "append":
        new = case["new"] if case["new"] <= 5 else case["new"] * 2 // 3
        n = case["B"] * new
        return {"bytes": n * Hkv * D * 2 * (2 + 1) + 16 * case["B"] * Hkv, "flops": 4 * n * Hkv * D}
    if op == "cache":
        B, H, T = case["B"], case["H"], case["T"]
        mean = max(1, case["context"] * 5 // 8)
        seen = min(mean, case["window"] + case["sinks"] + T - 1)
        return {"bytes": 2 * B * seen * Hkv * D + 4 * B * H * T * D + 4 * B * H * T,
                "flops": 4 * B * H * T * D * seen}
    if op == "fork":
        # each row of the table once, the reference counts read and written, most children's last pages copied
        rows, M = case["rows"], case["new_rows"]
        width = (case["context"] + case["reserve"] + case["page"] - 1) // case["page"]
        n_pages = rows * width + M * ((case["reserve"] + case["page"] - 1) // case["page"] + 2)
        copies = max(0, M - rows) + min(rows, M) // 3
        return {"bytes": 4 * (rows + M) * width + 8 * n_pages + 2 * copies * page_bytes, "flops": M * width}
    moved = case["pages"] * case["live"] * (1 - case["live"])
    return {"bytes": int(2 * moved * page_bytes) + 12 * case["pages"] + 8 * int(case["pages"] * case["live"]), "flops": case["pages"]}


# ---- the operators' definitions in 64 bits --------------------------------------------------------------------------

def _exact_window(case, s):
    q, k, v = (s[n].double() for n in ("q", "k", "v"))
    B, H, S, D = q.shape
    G = H // case["Hkv"]
    out, lse = s["out"].double().clone(), s["lse"].double().clone()
    c = torch.arange(S, device="cuda")
    step = max(1, min(S, 2048))
    for b in range(B):
        n = S if s["lengths"] is None else int(s["lengths"][b])
        for r0 in range(0, n, step):
            r = torch.arange(r0, min(n, r0 + step), device="cuda")
            # columns that any of these rows can see: the first tokens, and from the first row's window on
            lo = max(0, r0 - case["window"] + 1)
            cols = torch.cat([c[:min(case["sinks"], lo)], c[lo:int(r[-1]) + 1]])
            see = (cols <= r[:, None]) & ((cols > r[:, None] - case["window"]) | (cols < case["sinks"]))
            for h in range(H):
                score = q[b, h, r] @ k[b, h // G, cols].T / math.sqrt(D)
                score[~see] = -math.inf
                total = torch.logsumexp(score, -1)
                out[b, h, r] = torch.exp(score - total[:, None]) @ v[b, h // G, cols]
                lse[b, h, r] = total
    return out, lse


def _round_e4m3(x):
    """Nearest E4M3 value, ties to even, saturating at 448: steps of 2^-3 of the binade, of 2^-9 below 2^-6."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_append(case, s):
    page = case["page"]
    table, starts, lengths = s["table"].tolist(), s["starts"].tolist(), s["lengths"].tolist()
    got = {}
    for name in ("k", "v"):
        value = s[name].view(torch.float8_e4m3fn).double()
        scale = s[name + "_scale"].double()
        new = s[name + "_new"].double()
        for b, held in enumerate(lengths):
            t, end = starts[b], starts[b + 1]
            while t < end:
                pos = held + t - starts[b]
                at, slot = table[b][pos // page], pos % page
                n = min(page - slot, end - t)
                x = new[t:t + n].transpose(0, 1)             # [Hkv, n, D]
                amax = x.abs().amax((1, 2)).clamp(min=2.0 ** -100)
                want = torch.exp2(torch.ceil(torch.log2(amax / 448)))
                if slot:
                    want = torch.maximum(want, scale[at])
                    value[at] = _round_e4m3(value[at] * (scale[at] / want)[:, None, None])
                value[at, :, slot:slot + n] = _round_e4m3(x / want[:, None, None])
                scale[at] = want
                t += n
        got[name], got[name + "_scale"] = value, scale
    return [got["k"], got["v"], got["k_scale"], got["v_scale"]]


def _exact_cache(case, s):
    q = s["q"].double()
    B, H, T, D = q.shape
    G, page = H // case["Hkv"], case["page"]
    out, lse = torch.zeros_like(q), torch.zeros(B, H, T, device="cuda", dtype=torch.float64)
    for b, n in enumerate(s["lengths"].tolist()):
        lo = max(0, n - T - case["window"] + 1)
        pos = torch.arange(n, device="cuda")
        pos = pos[(pos < case["sinks"]) | (pos >= lo)]
        at = s["table"][b][pos // page].long()
        k, v = (s[x].view(torch.float8_e4m3fn)[at, :, pos % page].double() * s[x + "_scale"][at].double()[..., None] for x in ("k", "v"))
        for t in range(T):
            p = n - T + t
            if p < 0:
                lse[b, :, t] = -math.inf
                continue
            see = (pos <= p) & ((pos > p - case["window"]) | (pos < case["sinks"]))
            for h in range(case["Hkv"]):
                score = q[b, h * G:(h + 1) * G, t] @ k[see, h].T / math.sqrt(D)
                total = torch.logsumexp(score, -1)
                out[b, h * G:(h + 1) * G, t] = torch.exp(score - total[:, None]) @ v[see, h]
                lse[b, h * G:(h + 1) * G, t] = total
    return out, lse


def _exact_fork(case, s):
    page, reserve = case["page"], case["reserve"]
    table, lengths, parents = s["table"].tolist(), s["lengths"].tolist(), s["parents"].tolist()
    free = [i for i, r in enumerate(s["refs"].tolist()) if r == 0]
    width, n_pages = len(table[0]), s["refs"].numel()
    new, new_lengths, refs, used, copies, took = [], [], [0] * n_pages, 0, [], set()
    for p in parents:
        row = [-1] * width
        if not 0 <= p < len(table):
            new.append(row)
            new_lengths.append(0)
            continue
        n = lengths[p]
        held, total = -(-n // page), -(-(n + reserve) // page)
        for c in range(held):
            if c * page < case["sinks"] or (c + 1) * page - 1 > n - case["window"]:
                row[c] = table[p][c]
        copy = n % page != 0 and p in took and row[held - 1] >= 0
        took.add(p)
        need = copy + total - held
        if total > width or used + need > len(free):
            used += need if total <= width else 0
            new.append([-1] * width)
            new_lengths.append(-1)
            continue
        pages = free[used:used + need]
        used += need
        if copy:
            copies.append((row[held - 1], pages[0]))
            row[held - 1] = pages.pop(0)
        row[held:total] = pages
        for x in row:
            if x >= 0:
                refs[x] += 1
        new.append(row)
        new_lengths.append(n)
    whole = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    return [whole(new), whole(new_lengths), whole(refs), *_exact_copied(s, copies)]


def _exact_copied(s, copies):
    got = []
    for name in ("k", "v", "k_scale", "v_scale"):
        x = s[name].clone()
        if copies:
            src, dst = (torch.tensor(i, device="cuda") for i in zip(*copies))
            x[dst] = s[name][src]
        got.append(x.view(torch.float8_e4m3fn).double() if x.dtype == torch.uint8 else x.double())
    return got


def _exact_compact(case, s):
    refs, table = s["refs"].tolist(), s["table"].tolist()
    live = [i for i, r in enumerate(refs) if r > 0]
    holes = [i for i in range(len(live)) if refs[i] == 0]
    page_map = [-1] * len(refs)
    new_refs = [0] * len(refs)
    copies = []
    for i in live:
        to = i
        if i >= len(live):
            to = holes[len(copies)]
            copies.append((i, to))
        page_map[i] = to
        new_refs[to] = refs[i]
    whole = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    return [whole([[page_map[x] if x >= 0 else -1 for x in row] for row in table]), whole(new_refs), whole(page_map),
            whole([len(live)]), *_exact_copied(s, copies)]


EXACT = {"window": _exact_window, "append": _exact_append, "cache": _exact_cache, "fork": _exact_fork, "compact": _exact_compact}


def exact(case, seed):
    if case["op"] == "window" and case["B"] * case["H"] * case["S"] > (1 << 21) * 4:
        return None                                          # too many small products one after the other
    return EXACT[case["op"]](case, prepare(case, seed))
