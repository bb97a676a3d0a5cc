"""The operators of a layer that attends to whole sequences in float64 on the CPU, from their formulas."""
import math

import torch

from tests import _mixers_ref as mixers

TOP = 448.0


def rows(offsets):
    return [slice(int(a), int(b)) for a, b in zip(offsets[:-1], offsets[1:])]


def packed(q, k, v, offsets, scale=None):
    """(o, lse) of q [N,Hq,d], k, v [N,Hk,d]; rows of no sequence are 0 and -inf and are not read."""
    o, lse = [], torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64)
    for r in rows(offsets):
        n = r.stop - r.start
        if n:
            oi, li = mixers.window(q[None, r], k[None, r], v[None, r], n, 0, scale)
            o.append(oi[0])
            lse[:, r] = li[0].detach()
    last = int(offsets[-1])
    return torch.cat(o + [0.0 * q[last:]]), lse


def packed_bounds(q, k, v, do, offsets, scale=None, u=2.0 ** -8, acc=2.0 ** -20):
    out = {n: torch.zeros_like(x) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", k))}
    for r in rows(offsets):
        n = r.stop - r.start
        if n:
            for name, e in mixers.window_bounds(q[None, r], k[None, r], v[None, r], do[None, r], n, 0, scale, u=u, acc=acc).items():
                out[name][r] = e[0]
    return out


# ---- the cache in 8 bits -----------------------------------------------------------------------
E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()      # every number of the type
GRID = torch.sort(E4M3[:0x7f]).values                                               # 0 .. 448, 127 of them


def nearest(x):
    """The nearest e4m3 number, ties to the one with an even code, from the list of all; NaN stays."""
    a = x.abs().clamp(max=TOP)
    hi = torch.searchsorted(GRID, torch.nan_to_num(a, nan=0.0)).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    down, up = a - GRID[lo], GRID[hi] - a
    take = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    y = torch.where(x < 0, -GRID[take], GRID[take])
    return torch.where(x.isnan(), x, y)


def scale_of(x):
    """The smallest 2^e, e from -40 to 40, with max |finite x| <= 448 2^e."""
    big = float(x[x.isfinite()].abs().max()) if x.isfinite().any() else 0.0
    e = -40
    while e < 40 and big > TOP * 2.0 ** e:
        e += 1
    return 2.0 ** e


def turned(x, table, pos, grid_w=0, prefix=0, half=False):
    """One token's heads [H,d] turned for its position, in float64 from the table's fp32 numbers."""
    n = x.shape[-1] // 2
    if grid_w:
        j = pos - prefix
        if j < 0:
            return x.clone()
        last = table.shape[0] - 1
        t = torch.cat((table[min(j // grid_w, last)], table[min(j % grid_w, last)])).double()
    else:
        t = table[min(pos, table.shape[0] - 1)].double()
    c, s = t[:, 0], t[:, 1]
    if half:
        a, b = x[..., :n], x[..., n:]
        return torch.cat((a * c - b * s, a * s + b * c), -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)


def append(k, v, cache, block_table, pos, offsets=None, table=None, grid_w=0, prefix=0, half=False):
    """cache: dict of k_pages, v_pages (float64 numbers of the type) and k_scales, v_scales; changed in place.
    Page by page and head by head, as the definition reads."""
    P, Hk, page, d = cache["k_pages"].shape
    offsets = list(range(k.shape[0] + 1)) if offsets is None else offsets
    for b, r in enumerate(rows(offsets)):
        first, n = int(pos[b]), r.stop - r.start
        if first < 0 or n == 0:
            continue
        for j in range(first // page, (first + n - 1) // page + 1):
            if j >= block_table.shape[1] or not 0 <= int(block_table[b, j]) < P:
                continue
            at = int(block_table[b, j])
            lo, hi = max(first, j * page), min(first + n, (j + 1) * page)
            new = slice(lo - j * page, hi - j * page)
            for name, x in (("k", k), ("v", v)):
                x = x[r.start + lo - first: r.start + hi - first].double()
                if name == "k" and table is not None:
                    x = torch.stack([turned(x[i], table, lo + i, grid_w, prefix, half) for i in range(hi - lo)])
                x = x.float().double()
                pages, scales = cache[name + "_pages"], cache[name + "_scales"]
                for h in range(Hk):
                    s = scale_of(x[:, h])
                    if new.start > 0:
                        was = float(scales[at, h])
                        s = max(s, was)
                        if s > was:
                            pages[at, h, : new.start] = nearest(pages[at, h, : new.start] * (was / s))
                    scales[at, h] = s
                    pages[at, h, new] = nearest(x[:, h] / s)


def seen_at(cache, block_table, b, pos):
    """The tokens 0 .. pos of a sequence that stand in pages of the pool."""
    P, _, page, _ = cache["k_pages"].shape
    return [i for i in range(min(pos + 1, block_table.shape[1] * page)) if 0 <= int(block_table[b, i // page]) < P]


def seen_scale(cache, block_table, b, i, h):
    return cache["v_scales"][int(block_table[b, i // cache["k_pages"].shape[2]]), h]


def seen_tokens(cache, name, block_table, b, pos, h):
    """Their keys or values."""
    _, _, page, d = cache["k_pages"].shape
    out = []
    for i in seen_at(cache, block_table, b, pos):
        at = int(block_table[b, i // page])
        out.append(cache[name + "_pages"][at, h, i % page] * cache[name + "_scales"][at, h])
    return torch.stack(out) if out else torch.zeros(0, d, dtype=torch.float64)


def paged(q, cache, block_table, pos, scale=None, u=0.0, acc=2.0 ** -20):
    """(o, lse, bound of o): the bound for weights that carry a relative error of u and exponents one of acc.  A weight
    is rounded where it stands beside its value's 8-bit number, times the value's scale, with the largest at 2^11 or more:
    below 2^-14 fp16 has steps of 2^-24, so the error is at least up to 2^-25, 2^-36 of the largest."""
    B, Hq, d = q.shape
    G = Hq // cache["k_pages"].shape[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    o, lse, err = torch.zeros_like(q), torch.full((B, Hq), -math.inf, dtype=torch.float64), torch.zeros_like(q)
    for b in range(B):
        for h in range(Hq):
            if h % G == 0:
                k, v = (seen_tokens(cache, n, block_table, b, int(pos[b]), h // G) for n in ("k", "v"))
            if len(k):
                x = k @ q[b, h] * scale
                p = torch.softmax(x, 0)
                o[b, h], lse[b, h] = p @ v, torch.logsumexp(x, 0)
                e = u + acc * (2 + (k.abs() @ q[b, h].abs()) * abs(scale) + x.abs().max())
                s = torch.stack([seen_scale(cache, block_table, b, i, h // G) for i in seen_at(cache, block_table, b, int(pos[b]))])
                err[b, h] = (p * e) @ v.abs() + 2.0 ** -36 * (p * s).max() * (v.abs() / s[:, None]).sum(0)
    return o, lse, err
