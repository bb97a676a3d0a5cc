"""The operators of a layer that attends to whole sequences, as cases to be measured.

Three operators, each over its real range: causal attention over packed sequences (``packed``, forward
and gradient), appending rotated keys and values to a paged cache in 8 bits (``append``) and attention of
one new token per sequence over that cache (``paged``).  Shapes are those of the workloads in
``paper_2507_01652_b200/workloads.py``: layers of 4 to 24 heads of 32 or 64 channels over images of
16x16 to 96x96 tokens, with or without one class token in front.

``run`` computes an operator in plain torch operations in 32 bits (the rotation, whose results are
rounded to 8 bits, in 64), or, where ``own`` is set, by this package's calls.  ``exact`` is the
definition in 64 bits, sequence by sequence.
"""
import math

import torch

own = False

_BF16, _F32 = "bf16", "f32"
_LOW, _HIGH = -40, 40              # exponents that a page's scale can have
_TOP = 448.0                       # the largest number of the 8-bit type (e4m3)


# ---------------------------------------------------------------------------------------------
# cases: sequence b of S has lo + (hi - lo) b / (S - 1) tokens
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # a training step of the small fp32 layer (4 heads of 32 channels) on three short sequences
        dict(name="packed train 3x256 f32", op="packed", mode="train", dtype=_F32, S=3, lo=31, hi=256, tail=0, Hq=4, Hk=4, d=32),
        # a training step of the width-768 layer on 32 images of 16x16 tokens and their class token
        dict(name="packed train 32x257x12", op="packed", mode="train", dtype=_BF16, S=32, lo=257, hi=257, tail=0, Hq=12, Hk=12, d=64),
        # prefill of 64 unfinished images of up to 24x24 tokens, four query heads to a key head, in a buffer with room left
        dict(name="packed prefill 64x577x16", op="packed", mode="forward", dtype=_BF16, S=64, lo=1, hi=577, tail=96, Hq=16, Hk=4, d=64),
        # prefill of one 96x96 image, 24 heads
        dict(name="packed prefill 1x9217x24", op="packed", mode="forward", dtype=_BF16, S=1, lo=9217, hi=9217, tail=0, Hq=24, Hk=8, d=64),
        # a training step on images of four resolutions, packed without padding
        dict(name="packed train 4x9217x24", op="packed", mode="train", dtype=_BF16, S=4, lo=257, hi=9217, tail=0, Hq=24, Hk=8, d=64),
        # one generation step of the width-1280 layer: a token of every sequence into its page
        dict(name="append step 256x20", op="append", mode="step", dtype=_BF16, S=256, lo=1, hi=1, first=576, Hq=20, Hk=20, d=64,
             page=16, pages=37, grid_w=24, prefix=1, half=False),
        # the prompts of a batch of 24x24 images, some of them continued in the middle of a page
        dict(name="append prompts 64x577x16", op="append", mode="prompt", dtype=_BF16, S=64, lo=1, hi=577, first=40, Hq=16, Hk=4, d=64,
             page=32, pages=20, grid_w=24, prefix=1, half=True),
        # the prompts of eight 96x96 images, 24 query and 8 key heads
        dict(name="append prompts 8x9217x24", op="append", mode="prompt", dtype=_BF16, S=8, lo=9217, hi=9217, first=0, Hq=24, Hk=8, d=64,
             page=64, pages=145, grid_w=96, prefix=1, half=False),
        # one generation step of the small fp32 layer, three sequences
        dict(name="paged step 3x4 f32", op="paged", mode="step", dtype=_F32, S=3, lo=57, hi=257, Hq=4, Hk=4, d=32, page=16, pages=17),
        # one generation step of the width-1280 layer, sequences at every stage of a 24x24 image
        dict(name="paged step 256x20", op="paged", mode="step", dtype=_BF16, S=256, lo=0, hi=577, Hq=20, Hk=20, d=64, page=16, pages=37),
        # two long sequences: few rows, a long axis
        dict(name="paged step 2x24 long", op="paged", mode="step", dtype=_BF16, S=2, lo=9217, hi=9217, Hq=24, Hk=8, d=64, page=64, pages=145),
        # one generation step of 64 sequences at every stage of a 96x96 image
        dict(name="paged step 64x24", op="paged", mode="step", dtype=_BF16, S=64, lo=1, hi=9217, Hq=24, Hk=8, d=64, page=64, pages=145),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("packed", "packed", "append", "paged"))
    dtype = _BF16 if rng.random() < 0.8 else _F32
    d = rng.choice((32, 64, 64, 64))
    Hk = _log_int(rng, 1, 24)
    Hq = Hk * rng.choice([g for g in (1, 1, 2, 3, 4, 6, 8) if Hk * g <= 24])
    if op == "packed":
        # the fp32 form does a fortieth of the largest case's products, as its layers do
        most = 24 * 134000000 // (40 if dtype == _F32 else 1)
        hi = _log_int(rng, 1, min(9217, int(math.sqrt(most / Hq))))
        lo = rng.choice((hi, rng.randint(0, hi)))
        S = _log_int(rng, 1, max(1, min(256, most // (Hq * hi * hi), 131072 // hi)))
        mode = rng.choice(("forward", "train", "train"))
        return dict(op=op, mode=mode, dtype=dtype, S=S, lo=lo, hi=hi, tail=rng.choice((0, 0, rng.randint(1, 300))), Hq=Hq, Hk=Hk, d=d)
    page = rng.choice((16, 32, 64, 128))
    if op == "append":
        mode = rng.choice(("step", "prompt"))
        hi = 1 if mode == "step" else _log_int(rng, 1, 9217)
        lo = hi if mode == "step" else rng.choice((hi, rng.randint(0, hi)))
        first = rng.choice((0, rng.randint(0, 1000)))
        most = 8 * 9217 * 32 * 64 // (2 if dtype == _F32 else 1)
        S = _log_int(rng, 1, max(1, min(256, most // (hi * (Hq + Hk) * d), most // ((hi + first) * Hk * d))))
        return dict(op=op, mode=mode, dtype=dtype, S=S, lo=lo, hi=hi, first=first, Hq=Hq, Hk=Hk, d=d, page=page,
                    pages=-(-(hi + first) // page), grid_w=rng.choice((0, 16, 24, 96, rng.randint(2, 100))),
                    prefix=rng.choice((0, 1, 3)), half=rng.random() < 0.5)
    hi = _log_int(rng, 1, 9217)
    lo = rng.choice((hi, rng.randint(0, hi)))
    S = _log_int(rng, 1, max(1, min(256, 64 * 9217 * 8 * 64 // (hi * Hk * d))))
    return dict(op=op, mode="step", dtype=dtype, S=S, lo=lo, hi=hi, Hq=Hq, Hk=Hk, d=d, page=page, pages=-(-hi // page))


# ---------------------------------------------------------------------------------------------
# what a case's user has in hand
# ---------------------------------------------------------------------------------------------
def _lengths(c):
    S, lo, hi = c["S"], c["lo"], c["hi"]
    return [lo + (hi - lo) * b // (S - 1) for b in range(S)] if S > 1 else [hi]


def _firsts(c):
    """The position of each sequence's first new token: spread over 0 .. first."""
    S, n = c["S"], c["first"]
    return [n * ((7 * b) % S) // max(1, S - 1) for b in range(S)] if S > 1 else [n]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _table_rows(c):
    last = c["first"] + c["hi"]
    return max(c["grid_w"], last // c["grid_w"] + 1) if c["grid_w"] else last + 1


def _table(c):
    """cos and sin of position x 10000^(-m / pairs), from angles in 64 bits, as fp32 [rows, pairs, 2]."""
    pairs = c["d"] // (4 if c["grid_w"] else 2)
    freq = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -torch.arange(pairs, dtype=torch.float64) / pairs)
    a = torch.arange(_table_rows(c), dtype=torch.float64)[:, None] * freq[None, :]
    return torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32)


def _scale_of(amax):
    """The smallest power of two 2^e, e from _LOW to _HIGH, whose 448-fold is not below amax (fp32)."""
    m, e = torch.frexp(amax)                                    # amax = m 2^e, m from 1/2
    e = torch.where(m <= 0.875, e - 9, e - 8)                   # 448 = 0.875 x 2^9
    e = torch.where(amax > 0, e, torch.full_like(e, _LOW)).clamp(_LOW, _HIGH)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _to_8(x):
    return x.clamp(-_TOP, _TOP).to(torch.float8_e4m3fn)


_contexts = []


def _context():
    if not _contexts:
        from paper_2507_01652_b200 import binding
        _contexts.append(binding.Lasad(torch.cuda.current_device()))
    return _contexts[0]


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == _BF16 else torch.float32
    s = dict(case=c)

    def normal(*shape, dtype=dt, std=1.0):
        return torch.randn(*shape, generator=g, device=dev).mul_(std).to(dtype)

    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)   # noqa: E731
    S, Hq, Hk, d = c["S"], c["Hq"], c["Hk"], c["d"]
    lengths = _lengths(c)
    if c["op"] == "packed":
        at = _starts(lengths)
        N = max(1, at[-1] + c["tail"])
        s["q"], s["k"], s["v"] = normal(N, Hq, d, std=1.5), normal(N, Hk, d), normal(N, Hk, d)
        s["offsets"] = ints(at)
        if c["mode"] == "train":
            s["do"] = normal(N, Hq, d)
    else:
        page, P = c["page"], S * c["pages"] + 3                 # (a pool with three pages that nobody has)
        s["block_table"] = torch.randperm(P, generator=g, device=dev)[: S * c["pages"]].to(torch.int32).view(S, c["pages"]).contiguous()
        # a cache in use: values of the same distribution, each page with the scale of its largest
        for n in ("k", "v"):
            x = normal(P, Hk, page, d, dtype=torch.float32, std=1.0 if n == "k" else 0.5)
            scale = _scale_of(x.abs().amax(dim=(2, 3)))
            s[n + "_pages"], s[n + "_scales"] = _to_8(x / scale[:, :, None, None]), scale
            del x
        if c["op"] == "append":
            at = _starts(lengths)
            N = max(1, at[-1])
            s["k"], s["v"], s["q"] = normal(N, Hk, d, std=1.2), normal(N, Hk, d, std=0.5), normal(N, Hq, d)
            s["table"] = _table(c).to(dev)
            s["pos"] = ints(_firsts(c))
            if c["mode"] == "prompt":
                s["offsets"] = ints(at)
        else:
            s["q"] = normal(S, Hq, d, std=1.5)
            s["pos"] = ints([n - 1 for n in lengths])
    if own:
        s["ctx"] = _context()
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state["ctx"], state, state["case"])
    return _PLAIN[op](state, state["case"])


def _own_packed(ctx, s, c):
    o, lse = ctx.lasad_packed_attention(s["q"], s["k"], s["v"], s["offsets"], want_lse=True)
    if c["mode"] == "forward":
        return dict(o=o, lse=lse)
    dq, dk, dv = ctx.lasad_packed_attention_backward(s["q"], s["k"], s["v"], o, lse, s["do"], s["offsets"])
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)


def _own_append(ctx, s, c):
    q = ctx.lasad_paged_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["block_table"],
                               s["pos"], offsets=s.get("offsets"), q=s["q"], table=s["table"], grid_w=c["grid_w"],
                               prefix_len=c["prefix"], half=c["half"])
    return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"], k_scales=s["k_scales"], v_scales=s["v_scales"])


def _own_paged(ctx, s, c):
    o, lse = ctx.lasad_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["block_table"],
                                       s["pos"], want_lse=True)
    return dict(o=o, lse=lse)


_OWN = dict(packed=_own_packed, append=_own_append, paged=_own_paged)


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _softmax(x):
    """Row softmax of masked scores (-inf where masked): (p, log of the sum); an empty row gives 0, -inf."""
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    n = p.sum(dim=-1, keepdim=True)
    return p / torch.where(n == 0, torch.ones_like(n), n), (m + torch.log(n)).squeeze(-1)


def _plain_packed(s, c):
    dt, dev = s["q"].dtype, s["q"].device
    N, Hq, d = s["q"].shape
    Hk = c["Hk"]
    G = Hq // Hk
    scale = 1 / math.sqrt(d)
    lengths, T = _lengths(c), max(_lengths(c))
    names = ("o", "dq", "dk", "dv") if c["mode"] == "train" else ("o",)
    out = {n: torch.zeros(N, Hk if n in ("dk", "dv") else Hq, d, dtype=dt, device=dev) for n in names}
    out["lse"] = torch.full((Hq, N), -math.inf, device=dev)
    if T == 0:
        return out
    at = _starts(lengths)
    # short sequences of like lengths (they ascend) side by side in padded batches that are at least half full
    groups = [[]]
    for b in reversed(range(len(lengths))):
        group = [lengths[i] for i in groups[-1] + [b]]
        if len(group) > 1 and (max(group) > 1024 or sum(n * n for n in group) * 2 < len(group) * max(group) ** 2):
            groups.append([])
        groups[-1].append(b)
    for group in groups:
        T = max(lengths[b] for b in group)
        if T == 0:
            continue
        first = torch.tensor([at[b] for b in group], device=dev)
        n = torch.tensor([lengths[b] for b in group], device=dev)
        t = torch.arange(T, device=dev)
        inside = t[None, :] < n[:, None]
        at_row = torch.where(inside, first[:, None] + t, torch.zeros_like(t))        # [B, T]
        B = len(group)
        rows = lambda x: x[at_row].float().view(B, T, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * T, d)   # noqa: E731
        back = lambda x: x.view(B, Hk, G, T, d).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, d)[inside].to(dt)        # noqa: E731
        q, k, v = rows(s["q"]), s["k"][at_row].float().transpose(1, 2), s["v"][at_row].float().transpose(1, 2)
        seen = ((t[None, :] <= t[:, None]) & inside[:, :, None] & inside[:, None, :]).view(B, 1, 1, T, T)
        x = (torch.matmul(q, k.transpose(2, 3)) * scale).view(B, Hk, G, T, T)
        p, lse = _softmax(x.masked_fill_(~seen, -math.inf))
        del x
        p = p.view(B, Hk, G * T, T)
        o = torch.matmul(p, v)
        to = at_row[inside]
        out["o"][to] = back(o)
        out["lse"][:, to] = lse.reshape(B, Hq, T).permute(1, 0, 2)[:, inside]
        if c["mode"] == "forward":
            continue
        do = rows(s["do"])
        out["dv"][to] = torch.matmul(p.transpose(2, 3), do).transpose(1, 2)[inside].to(dt)
        ds = p * (torch.matmul(do, v.transpose(2, 3)) - (do * o).sum(dim=-1, keepdim=True)) * scale
        out["dq"][to] = back(torch.matmul(ds, k))
        out["dk"][to] = torch.matmul(ds.transpose(2, 3), q).transpose(1, 2)[inside].to(dt)
    return out


def _turn(x, cos, sin, half):
    """Pairs of channels turned, in 64 bits, rounded to 32."""
    x = x.double()
    n = x.shape[-1] // 2
    x0, x1 = (x[..., :n], x[..., n:]) if half else (x[..., 0::2], x[..., 1::2])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    return (torch.cat((y0, y1), dim=-1) if half else torch.stack((y0, y1), dim=-1).flatten(-2)).float()


def _plain_append(s, c):
    dev, page, Hk, d = s["k"].device, c["page"], c["Hk"], c["d"]
    P = s["k_pages"].shape[0]
    # every token's sequence and position
    if "offsets" in s:
        i = torch.arange(s["k"].shape[0], device=dev)
        b = torch.searchsorted(s["offsets"][1:].contiguous(), i.int(), right=True)
        ours = b < c["S"]
        b = b.clamp(max=c["S"] - 1)
        pos = s["pos"][b].long() + i - s["offsets"][b]
    else:
        b, pos = torch.arange(c["S"], device=dev), s["pos"].long()
        ours = pos >= 0
    if c["grid_w"]:
        j = (pos - c["prefix"]).clamp(min=0)
        t = torch.cat((s["table"][j // c["grid_w"]], s["table"][j % c["grid_w"]]), dim=1)
        t = torch.where((pos >= c["prefix"])[:, None, None], t, torch.tensor([1.0, 0.0], device=dev))
    else:
        t = s["table"][pos]
    cos, sin = t[:, None, :, 0].double(), t[:, None, :, 1].double()
    q = _turn(s["q"], cos, sin, c["half"]).to(s["q"].dtype)
    at, slot = s["block_table"][b, pos // page].long(), pos % page
    at = torch.where(ours, at, torch.full_like(at, P))           # (a place behind the pool for rows of nobody)
    out = dict(q=q)
    first = torch.full((P + 1,), page, dtype=torch.long, device=dev).scatter_reduce_(0, at, slot, "amin")[:P]
    touched = (first < page).nonzero().squeeze(1)
    kept = torch.arange(page, device=dev)[None, :] < first[touched][:, None]         # tokens that were there
    for name in ("k", "v"):
        x = _turn(s["k"], cos, sin, c["half"]) if name == "k" else s["v"].float()
        pages, scales = s[name + "_pages"], s[name + "_scales"]
        amax = torch.zeros(P + 1, Hk, device=dev).scatter_reduce_(0, at[:, None].expand(-1, Hk), x.abs().amax(dim=-1), "amax")[touched]
        was = scales[touched]
        now = torch.where(first[touched][:, None] > 0, torch.maximum(was, _scale_of(amax)), _scale_of(amax))
        old = pages[touched]
        again = _to_8(old.float() * (was / now)[:, :, None, None])
        grown = kept[:, None, :, None] & (now > was)[:, :, None, None]
        pages.view(torch.uint8)[touched] = torch.where(grown, again.view(torch.uint8), old.view(torch.uint8))
        scales[touched] = now
        new = _to_8(x / torch.cat((scales, torch.ones(1, Hk, device=dev)))[at][:, :, None])
        pages.view(torch.uint8)[at[ours], :, slot[ours]] = new.view(torch.uint8)[ours]
        out.update({name + "_pages": pages, name + "_scales": scales})
    return out


def _plain_paged(s, c):
    S, Hq, d = s["q"].shape
    Hk, T = c["Hk"], c["pages"] * c["page"]
    at = s["block_table"].long()

    def whole(name):          # [S, Hk, T, d]
        x = s[name + "_pages"][at].float() * s[name + "_scales"][at][..., None, None]
        return x.transpose(1, 2).reshape(S, Hk, T, d)

    k = whole("k")
    x = torch.matmul(s["q"].float().view(S, Hk, Hq // Hk, d), k.transpose(2, 3)) / math.sqrt(d)
    del k
    seen = torch.arange(T, device=x.device) <= s["pos"][:, None]
    p, lse = _softmax(x.masked_fill_(~seen[:, None, None], -math.inf))
    return dict(o=torch.matmul(p, whole("v")).view(S, Hq, d).to(s["q"].dtype), lse=lse.view(S, Hq))


_PLAIN = dict(packed=_plain_packed, append=_plain_append, paged=_plain_paged)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    c = case
    e = 2 if c["dtype"] == _BF16 else 4
    S, Hq, Hk, d = c["S"], c["Hq"], c["Hk"], c["d"]
    lengths = _lengths(c)
    n = sum(lengths)
    if c["op"] == "packed":
        pairs = sum(m * (m + 1) // 2 for m in lengths)
        q, k, lse = n * Hq * d * e, n * Hk * d * e, n * Hq * 4
        train = c["mode"] == "train"
        # forward: q, k, v in, o out; training adds q, k, v, o, do in and dq, dk, dv out
        return dict(bytes=max(1, (2 * q + 2 * k + lse) + ((4 * q + 4 * k + lse) if train else 0)),
                    flops=pairs * Hq * d * (14 if train else 4))
    if c["op"] == "append":
        # k, v, q in, q out in their type; k, v out in a byte; a scale of every page and head touched
        pages = sum(-(-(f + m) // c["page"]) - f // c["page"] for f, m in zip(_firsts(c), lengths) if m)
        return dict(bytes=max(1, n * d * (2 * Hk * (e + 1) + 2 * Hq * e) + pages * Hk * 8), flops=n * (Hq + Hk) * d * 3)
    pages = sum(-(-m // c["page"]) for m in lengths)
    return dict(bytes=2 * n * Hk * d + pages * (Hk * 8 + 4) + S * Hq * (2 * d * e + 4), flops=4 * n * Hq * d)


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return dict(packed=_exact_packed, append=_exact_append, paged=_exact_paged)[case["op"]](s, case)


def _exact_packed(s, c):
    G, f, train = c["Hq"] // c["Hk"], c["d"] ** -0.5, c["mode"] == "train"
    q64 = lambda n: torch.zeros_like(s[n], dtype=torch.float64)   # noqa: E731
    out = dict(o=q64("q"), lse=torch.full((c["Hq"], s["q"].shape[0]), -math.inf, dtype=torch.float64, device=s["q"].device))
    if train:
        out.update(dq=q64("q"), dk=q64("k"), dv=q64("k"))
    at = 0
    for n in _lengths(c):
        own_rows = slice(at, at + n)
        at += n
        size = max(1, (1 << 24) // max(1, n))                     # rows at a time
        for h in range(c["Hq"] if n else 0):
            k, v = s["k"][own_rows, h // G].double(), s["v"][own_rows, h // G].double()
            for t0 in range(0, n, size):
                t = torch.arange(t0, min(n, t0 + size), device=k.device)
                here = slice(own_rows.start + t0, own_rows.start + t0 + len(t))
                m = t0 + len(t)                                   # keys that any of these rows sees
                x = s["q"][here, h].double() @ k[:m].T * f
                x[torch.arange(m, device=k.device)[None, :] > t[:, None]] = -math.inf
                z = torch.logsumexp(x, -1)
                a = torch.exp(x - z[:, None])
                out["o"][here, h], out["lse"][h, here] = a @ v[:m], z
                if train:
                    g = s["do"][here, h].double()
                    da = g @ v[:m].T
                    dx = a * (da - (a * da).sum(-1, keepdim=True)) * f
                    out["dq"][here, h] = dx @ k[:m]
                    seen = slice(own_rows.start, own_rows.start + m)
                    out["dk"][seen, h // G] += dx.T @ s["q"][here, h].double()
                    out["dv"][seen, h // G] += a.T @ g
    return out


def _nearest_8(x):
    """The nearest number of the 8-bit type (4 bits of significand, 2^-9 the smallest step), ties to even."""
    step = torch.full_like(x, 2.0 ** -9)
    for e in range(-5, 9):
        step = torch.where(x.abs() >= 2.0 ** e, 2.0 ** (e - 3), step)
    return (torch.round(x / step) * step).clamp(-_TOP, _TOP)


def _exact_append(s, c):
    page, d = c["page"], c["d"]
    n = d // 2
    to_c = (lambda v: torch.complex(v[..., :n], v[..., n:])) if c["half"] else (
        lambda v: torch.view_as_complex(v.unflatten(-1, (n, 2)).contiguous()))
    to_r = (lambda v: torch.cat((v.real, v.imag), -1)) if c["half"] else (lambda v: torch.view_as_real(v).flatten(-2))
    spins = torch.view_as_complex(s["table"].double().contiguous())
    out = {m: s[m].double() for m in ("k_pages", "v_pages", "k_scales", "v_scales")}
    out["q"] = torch.zeros_like(s["q"], dtype=torch.float64)
    at = 0
    for b, (start, m) in enumerate(zip(_firsts(c), _lengths(c))):
        rows = slice(at, at + m)
        at += m
        if m == 0:
            continue
        i = torch.arange(start, start + m, device=spins.device)
        if c["grid_w"]:
            j = i - c["prefix"]
            w = c["grid_w"]
            spin = torch.cat((spins[torch.div(j, w, rounding_mode="floor").clamp(min=0)], spins[j.remainder(w)]), 1)
            spin[j < 0] = 1
        else:
            spin = spins[i]
        turn = lambda x: to_r(to_c(x.double()) * spin[:, None])   # noqa: E731
        out["q"][rows] = turn(s["q"][rows])
        new = dict(k=turn(s["k"][rows]).float().double(), v=s["v"][rows].double())    # (32 bits go into the rounding to 8)
        # the pages from the one that the first new token falls into, as one run of tokens
        p0, p1 = start // page, (start + m - 1) // page
        ids = s["block_table"][b, p0:p1 + 1].long()
        before = start - p0 * page
        for name, x in new.items():
            was = out[name + "_scales"][ids]                                          # [pages, Hk]
            run = out[name + "_pages"][ids].transpose(1, 2).flatten(0, 1)             # [tokens, Hk, d]
            size = torch.zeros(len(ids) * page, c["Hk"], dtype=torch.float64, device=x.device)
            size[before:before + m] = x.abs().amax(-1)
            size = size.view(len(ids), page, -1).amax(1)
            now = torch.full_like(size, 2.0 ** _LOW)
            for e in range(_LOW, _HIGH):                                              # up to the first that is enough
                now = torch.where(size > _TOP * 2.0 ** e, 2.0 ** (e + 1), now)
            if before:
                now[0] = torch.maximum(now[0], was[0])
                run[:before] = _nearest_8(run[:before] * (was[0] / now[0])[:, None])
            run[before:before + m] = _nearest_8(x / now.repeat_interleave(page, 0)[before:before + m, :, None])
            out[name + "_scales"][ids] = now
            out[name + "_pages"][ids] = run.unflatten(0, (len(ids), page)).transpose(1, 2)
    return out


def _exact_paged(s, c):
    S, Hq, d = s["q"].shape
    G = Hq // c["Hk"]
    o = torch.zeros(S, Hq, d, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((S, Hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        ids = s["block_table"][b, : -(-n // c["page"])].long()
        k, v = ((s[m + "_pages"][ids].double() * s[m + "_scales"][ids].double()[..., None, None])
                .transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(G, dim=0) for m in ("k", "v"))
        x = torch.einsum("hd,hnd->hn", s["q"][b].double(), k) * d ** -0.5
        lse[b] = torch.logsumexp(x, -1)
        o[b] = torch.einsum("hn,hnd->hd", torch.exp(x - lse[b][:, None]), v)
    return dict(o=o, lse=lse)
