"""Plain references in float64 of the serving operators, from their definitions, for small problems."""
import math

import torch

NONE = 2 ** 31 - 1


def visible(p, j, window, sinks):
    """Whether the query at position p sees key j."""
    return j <= p and (j > p - window or j < sinks)


def mask(positions, n_keys, window, sinks):
    p = positions.to(torch.int64)[:, None]
    j = torch.arange(n_keys, dtype=torch.int64)[None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def attention(q, k, v, see, scale=None):
    """q [R, D], k, v [N, D], see [R, N]: (out [R, D], lse [R]) in float64; keys that a row does not see are left out of it, rows
    without a key give 0 and -inf."""
    q, k, v = q.double(), k.double(), v.double()
    scale = 1 / math.sqrt(q.shape[1]) if not scale else scale
    out = torch.zeros_like(q)
    lse = torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    used = see.any(0)
    k, v, see = k[used], v[used], see[:, used]
    s = (q @ k.T * scale).masked_fill(~see, -math.inf)
    some = see.any(1)
    lse[some] = torch.logsumexp(s[some], -1)
    out[some] = torch.exp(s[some] - lse[some][:, None]) @ v
    return out, lse


def value_of_codes(codes):
    return codes.view(torch.float8_e4m3fn).double()


def e4m3(x):
    """Nearest E4M3 value of float64 numbers, ties to even, saturating at 448; NaN stays."""
    x = x.clamp(-448, 448)                       # (infinities too)
    a = x.abs()
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -60))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def scale_for(a):
    """Smallest power of two s with a <= 448 s, a at least 2^-100."""
    a = max(float(a), 2.0 ** -100)
    s = 2.0 ** (math.frexp(a)[1] - 9)
    return s if a <= 448 * s else 2 * s


class Cache:
    """The cache in float64 on the CPU."""

    def __init__(self, k, v, k_scale, v_scale):
        self.value = [value_of_codes(k.cpu()), value_of_codes(v.cpu())]
        self.scale = [k_scale.cpu().double(), v_scale.cpu().double()]
        self.n_pages, self.heads, self.page, self.D = self.value[0].shape

    def page_at(self, table, b, j):
        e = int(table[b, j // self.page]) if j // self.page < table.shape[1] else -1
        return e if 0 <= e < self.n_pages else -1

    def append(self, new, table, lengths, starts):
        for which in (0, 1):
            x = new[which].cpu().double()
            for b in range(table.shape[0]):
                held, t0, t1 = int(lengths[b]), int(starts[b]), int(starts[b + 1])
                t = t0
                while t < t1:
                    j = held + t - t0
                    slot = j % self.page
                    n = min(self.page - slot, t1 - t)
                    e = self.page_at(table, b, j)
                    if e >= 0:
                        for h in range(self.heads):
                            rows = x[t:t + n, h]
                            a = rows[torch.isfinite(rows)].abs()
                            s = scale_for(a.max() if a.numel() else 0.0)
                            if slot:
                                old = float(self.scale[which][e, h])
                                s = max(s, old)
                                if s > old:
                                    self.value[which][e, h] = e4m3(self.value[which][e, h] * (old / s))
                            self.value[which][e, h, slot:slot + n] = e4m3(rows / s)
                            self.scale[which][e, h] = s
                    t += n

    def keys(self, table, b, n, h):
        """K, V [n, D] of head h and which of the n tokens have a page."""
        k, v = torch.zeros(n, self.D, dtype=torch.float64), torch.zeros(n, self.D, dtype=torch.float64)
        there = torch.zeros(n, dtype=torch.bool)
        for c in range(-(-n // self.page)):
            e = self.page_at(table, b, c * self.page)
            if e >= 0:
                at = slice(c * self.page, min(n, (c + 1) * self.page))
                m = at.stop - at.start
                k[at] = self.value[0][e, h, :m] * self.scale[0][e, h]
                v[at] = self.value[1][e, h, :m] * self.scale[1][e, h]
                there[at] = True
        return k, v, there


def cache_attention(cache, q, table, lengths, window, sinks, scale=None):
    """q [B, H, T, D] on the CPU: (out, lse) in float64."""
    B, H, T, D = q.shape
    out, lse = torch.zeros(B, H, T, D, dtype=torch.float64), torch.zeros(B, H, T, dtype=torch.float64)
    G = H // cache.heads
    for b in range(B):
        n = max(0, min(int(lengths[b]), table.shape[1] * cache.page))
        pos = n - T + torch.arange(T)
        for hk in range(cache.heads):
            k, v, there = cache.keys(table, b, n, hk)
            see = mask(pos, n, window, sinks) & there
            for h in range(hk * G, hk * G + G):
                out[b, h], lse[b, h] = attention(q[b, h], k, v, see, scale)
    return out, lse


def fork(table, lengths, refs, parents, page, n_pages, reserve, window, sinks):
    """(new_table, new_lengths, new_refs, copies [(from, to)]) as lists."""
    rows, width = len(table), len(table[0])
    free = [i for i, r in enumerate(refs) if r == 0]
    new, new_lengths, new_refs, copies, took, used, full = [], [], [0] * n_pages, [], set(), 0, False
    for p in parents:
        row = [-1] * width
        if not 0 <= p < rows:
            new.append(row); new_lengths.append(0)
            continue
        n = max(0, lengths[p])
        held, total = -(-n // page), -(-(n + reserve) // page)
        first = p not in took
        took.add(p)
        if total > width:
            new.append(row); new_lengths.append(-1)
            continue
        keep = [table[p][c] if (any(visible(q, j, window, sinks) for q in (n,) for j in range(c * page, (c + 1) * page)) and
                                0 <= table[p][c] < n_pages) else -1 for c in range(held)]
        copy = n % page != 0 and not first and keep[-1] >= 0
        need = total - held + copy
        if full or used + need > len(free):
            full = True
            new.append(row); new_lengths.append(-1)
            continue
        fresh = free[used:used + need]
        used += need
        if copy:
            copies.append((keep[-1], fresh[0]))
            keep[-1] = fresh.pop(0)
        row[:total] = keep + fresh
        for e in row:
            if e >= 0:
                new_refs[e] += 1
        new.append(row); new_lengths.append(n)
    return new, new_lengths, new_refs, copies


def compact(table, refs):
    live = [i for i, r in enumerate(refs) if r > 0]
    holes = [i for i in range(len(live)) if refs[i] <= 0]
    page_map = [i if r > 0 and i < len(live) else -1 for i, r in enumerate(refs)]
    movers = [i for i in live if i >= len(live)]
    for src, dst in zip(movers, holes):
        page_map[src] = dst
    new_refs = [0] * len(refs)
    for i in live:
        new_refs[page_map[i]] = refs[i]
    new_table = [[page_map[e] if 0 <= e < len(refs) else -1 for e in row] for row in table]
    return new_table, new_refs, page_map, len(live), list(zip(movers, holes))
