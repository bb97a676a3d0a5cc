"""The operators that stand beside LASAD in a hybrid stack, as cases to be measured.

Three operators, each over its real range: the gated linear recurrence with the spatial rule
(``scan``), the per-head norm of queries and keys with the grid rotation (``rope``) and attention
over a sliding window with leading tokens that stay visible (``window``).  Shapes are those of the
workloads in ``paper_2507_01652_b200/workloads.py``: layers of 12 to 24 heads of 64 channels over
grids of 16x16 to 96x96 tokens, with or without one class token in front.

``run`` computes an operator in plain torch operations in 32 bits, or, where ``own`` is set, by
this package's calls.  ``exact`` is the definition in 64 bits, token by token or head by head.
"""
import math

import torch

own = False

_BF16, _F32 = "bf16", "f32"


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # one generation step of a width-1280 recurrent layer, every sequence at its own position
        dict(name="scan step 256x1280", op="scan", mode="step", dtype=_BF16, B=256, T=1, C=1280, grid_w=16,
             prefix=1, tied=True, logits=True),
        # the small fp32 layer (4 heads of 32 channels, 16x16 grid): a training step where launches count
        dict(name="scan train 1x256x128 f32", op="scan", mode="train", dtype=_F32, B=1, T=256, C=128, grid_w=16,
             prefix=0, tied=True, logits=False),
        # one high-resolution image (96x96 and its class token) through a width-1536 layer: few channels, long
        dict(name="scan prefill 1x9217x1536", op="scan", mode="forward", dtype=_BF16, B=1, T=9217, C=1536,
             grid_w=96, prefix=1, tied=True, logits=True),
        # a training step of that layer on a batch of 8
        dict(name="scan train 8x9216x1536", op="scan", mode="train", dtype=_BF16, B=8, T=9216, C=1536, grid_w=96,
             prefix=0, tied=True, logits=True),
        # one generation step of the width-1280 layer: norm and rotation of one token a sequence
        dict(name="rope step 256x20", op="rope", mode="forward", dtype=_BF16, B=256, T=1, Hq=20, Hk=20, d=64,
             grid_w=16, prefix=1, ragged=True, half=False),
        # prefill of a batch of 24x24 images, four query heads to a key head
        dict(name="rope prefill 64x577x16", op="rope", mode="forward", dtype=_BF16, B=64, T=577, Hq=16, Hk=4, d=64,
             grid_w=24, prefix=1, ragged=False, half=False),
        # a training step on 64x64 images, 24 heads
        dict(name="rope train 8x4096x24", op="rope", mode="train", dtype=_BF16, B=8, T=4096, Hq=24, Hk=24, d=64,
             grid_w=64, prefix=0, ragged=False, half=True),
        # one generation step: a window of 4 grid rows of 16 and the class token, some sequences just begun
        dict(name="window step 256x20 w64", op="window", mode="step", dtype=_BF16, B=256, T=1, Hq=20, Hk=20, d=64,
             window=64, sinks=1, ragged=True),
        # the same for two long sequences with a wide window: few rows, a long axis
        dict(name="window step 2x24 w4096", op="window", mode="step", dtype=_BF16, B=2, T=1, Hq=24, Hk=8, d=64,
             window=4096, sinks=1, ragged=False),
        # prefill of a batch of 24x24 images, a window of 6 grid rows
        dict(name="window prefill 64x577x16", op="window", mode="forward", dtype=_BF16, B=64, T=577, Hq=16, Hk=16,
             d=64, window=144, sinks=1, ragged=False),
        # a small training batch of sequences of all lengths, an empty one among them
        dict(name="window train 5x257x12", op="window", mode="train", dtype=_BF16, B=5, T=257, Hq=12, Hk=4, d=64,
             window=37, sinks=3, ragged=True),
        # a training step on one 96x96 image, 24 heads, a window of 16 grid rows
        dict(name="window train 1x9217x24", op="window", mode="train", dtype=_BF16, B=1, T=9217, Hq=24, Hk=8, d=64,
             window=1536, sinks=1, ragged=False),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(("scan", "rope", "window"))
    dtype = _BF16 if rng.random() < 0.8 else _F32
    prefix = rng.choice((0, 1, 1, 3))
    grid_w = rng.choice((0, 16, 24, 64, 96, rng.randint(2, 100)))
    if op == "scan":
        mode = rng.choice(("step", "forward", "train", "train"))
        C = 8 * _log_int(rng, 4, 192)
        most = 8 * 9216 * 1536 // (2 if dtype == _F32 else 1)
        T = 1 if mode == "step" else _log_int(rng, 1, 9217)
        B = _log_int(rng, 1, max(1, min(256, most // (T * C))))
        return dict(op=op, mode=mode, dtype=dtype, B=B, T=T, C=C, grid_w=grid_w, prefix=prefix,
                    tied=rng.random() < 0.7, logits=rng.random() < 0.6)
    d = rng.choice((32, 64, 64, 64))
    Hk = _log_int(rng, 1, 24)
    Hq = Hk * rng.choice([g for g in (1, 1, 2, 3, 4, 6, 8) if Hk * g <= 24])
    if op == "rope":
        mode = rng.choice(("forward", "train"))
        T = rng.choice((1, _log_int(rng, 1, 9217)))
        most = 8 * 4096 * 48 * 64 // (2 if dtype == _F32 else 1)
        B = _log_int(rng, 1, max(1, min(256, most // (T * (Hq + Hk) * d))))
        return dict(op=op, mode=mode, dtype=dtype, B=B, T=T, Hq=Hq, Hk=Hk, d=d, grid_w=grid_w, prefix=prefix,
                    ragged=rng.random() < 0.5, half=rng.random() < 0.5)
    mode = rng.choice(("step", "forward", "train", "train"))
    window = _log_int(rng, 1, 4096)
    ragged = rng.random() < 0.5
    if mode == "step":
        B = _log_int(rng, 1, max(1, min(256, 256 * 20 * 4096 // (window * Hk * 8))))
        return dict(op=op, mode=mode, dtype=dtype, B=B, T=1, Hq=Hq, Hk=Hk, d=d, window=window, sinks=prefix,
                    ragged=ragged)
    # the fp32 form does a fortieth of the largest case's products, as its layers do
    most = 24 * 9217 * 9217 // (40 if dtype == _F32 else 2)
    T = _log_int(rng, 1, min(9217, int(math.sqrt(most / Hq))))
    B = _log_int(rng, 1, max(1, min(64, most // (Hq * T * T))))
    return dict(op=op, mode=mode, dtype=dtype, B=B, T=T, Hq=Hq, Hk=Hk, d=d, window=window, sinks=prefix,
                ragged=ragged)


# ---------------------------------------------------------------------------------------------
# what a case's user has in hand
# ---------------------------------------------------------------------------------------------
def _spread(B, lo, hi):
    """B whole numbers from lo to hi, evenly: the lengths or positions of a ragged batch."""
    return [lo + (hi - lo) * b // max(1, B - 1) for b in range(B)] if B > 1 else [hi]


def _positions(case):
    """The position of each sequence's token (steps): -1 is a sequence that has ended."""
    if case["op"] == "window":
        last = case["window"] + case["sinks"] + case["window"] // 3
        return _spread(case["B"], -1, last) if case["ragged"] else [last] * case["B"]
    return _spread(case["B"], 0, 256)


def _lengths(case):
    return _spread(case["B"], 0, case["T"]) if case["ragged"] else None


def _table_rows(case):
    last = 256 + case["T"]
    if case["grid_w"] == 0:
        return last + 1
    return max(case["grid_w"], last // case["grid_w"] + 1)


def _angles(case):
    """Rotation angles in 64 bits, [rows, pairs]: position x 10000^(-m / pairs)."""
    pairs = case["d"] // (4 if case["grid_w"] else 2)
    freq = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -torch.arange(pairs, dtype=torch.float64) / pairs)
    return torch.arange(_table_rows(case), dtype=torch.float64)[:, None] * freq[None, :]


_contexts = []


def _context():
    if not _contexts:
        from paper_2507_01652_b200 import binding
        _contexts.append(binding.Lasad(torch.cuda.current_device()))
    return _contexts[0]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == _BF16 else torch.float32
    s = dict(case=case)

    def normal(*shape, dtype=dt, mean=0.0, std=1.0):
        return torch.randn(*shape, generator=g, device=dev).mul_(std).add_(mean).to(dtype)

    B, T = case["B"], case["T"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)   # noqa: E731
    if case["op"] == "scan":
        shape = (B, case["C"]) if case["mode"] == "step" else (B, T, case["C"])
        s["x"] = normal(*shape)
        # forget gates of trained layers sit near 1: logits around 2
        z = normal(*shape, dtype=torch.float32, mean=2.0)
        s["gate"] = (z if case["logits"] else torch.sigmoid(z)).to(dt)
        s["h_in"] = normal(B, case["C"], dtype=torch.float32)
        if case["mode"] == "step":
            s["pos"] = ints(_positions(case))
        if case["mode"] == "train":
            s["dy"] = normal(*shape)
            s["dh_out"] = normal(B, case["C"], dtype=torch.float32)
    elif case["op"] == "rope":
        Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
        s["q"], s["k"] = normal(B, T, Hq, d), normal(B, T, Hk, d, std=2.0)
        s["wq"], s["wk"] = (normal(d, dtype=torch.float32, mean=1.0, std=0.1) for _ in range(2))
        a = _angles(case)
        s["table"] = torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32).to(dev)
        if case["ragged"]:
            s["pos"] = ints(_spread(B, 0, 256))
        if case["mode"] == "train":
            s["dq_out"], s["dk_out"] = normal(B, T, Hq, d), normal(B, T, Hk, d)
    else:
        Hq, Hk, d = case["Hq"], case["Hk"], case["d"]
        if case["mode"] == "step":
            slots = case["sinks"] + case["window"]
            s["q"], s["k"], s["v"] = normal(B, Hq, d, std=1.5), normal(B, Hk, d), normal(B, Hk, d)
            s["k_cache"], s["v_cache"] = normal(B, slots, Hk, d), normal(B, slots, Hk, d)
            s["pos"] = ints(_positions(case))
        else:
            s["q"], s["k"], s["v"] = normal(B, T, Hq, d, std=1.5), normal(B, T, Hk, d), normal(B, T, Hk, d)
            if case["ragged"]:
                s["lengths"] = ints(_lengths(case))
            if case["mode"] == "train":
                s["do"] = normal(B, T, Hq, d)
    if own:
        s["ctx"] = _context()
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(state):
    op, mode = state["case"]["op"], state["case"]["mode"]
    if own:
        return _OWN[op](state["ctx"], state, state["case"], mode)
    return _PLAIN[op](state, state["case"], mode)


def _own_scan(ctx, s, c, mode):
    kw = dict(grid_w=c["grid_w"], prefix_len=c["prefix"], tied=c["tied"], logits=c["logits"])
    if mode == "step":
        y, h = ctx.lasad_scan_step(s["x"], s["gate"], s["h_in"], pos=s["pos"], h_out=torch.empty_like(s["h_in"]), **kw)
        return dict(y=y, h=h)
    y, h, saved = ctx.lasad_scan_forward(s["x"], s["gate"], h_in=s["h_in"], save=mode == "train", **kw)
    if mode == "forward":
        return dict(y=y, h=h)
    dx, dgate, dh_in = ctx.lasad_scan_backward(s["x"], s["gate"], saved, s["dy"], dh_out=s["dh_out"], **kw)
    return dict(y=y, h=h, dx=dx, dgate=dgate, dh_in=dh_in)


def _own_rope(ctx, s, c, mode):
    kw = dict(q_weight=s["wq"], k_weight=s["wk"], grid_w=c["grid_w"], prefix_len=c["prefix"], pos=s.get("pos"),
              half=c["half"], eps=1e-6)
    q, k = ctx.lasad_qk_norm_rope(s["q"], s["k"], s["table"], **kw)
    if mode == "forward":
        return dict(q=q, k=k)
    dq, dk, dwq, dwk = ctx.lasad_qk_norm_rope_backward(s["q"], s["k"], s["table"], s["dq_out"], s["dk_out"], **kw)
    return dict(q=q, k=k, dq=dq, dk=dk, dwq=dwq, dwk=dwk)


def _own_window(ctx, s, c, mode):
    if mode == "step":
        o = ctx.lasad_window_attention_step(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["pos"],
                                            c["window"], c["sinks"])
        return dict(o=o, k_cache=s["k_cache"], v_cache=s["v_cache"])
    kw = dict(window=c["window"], sinks=c["sinks"], lengths=s.get("lengths"))
    o, lse = ctx.lasad_window_attention(s["q"], s["k"], s["v"], want_lse=True, **kw)
    if mode == "forward":
        return dict(o=o, lse=lse)
    dq, dk, dv = ctx.lasad_window_attention_backward(s["q"], s["k"], s["v"], o, lse, s["do"], **kw)
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv)


_OWN = dict(scan=_own_scan, rope=_own_rope, window=_own_window)


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _ends_row(i, c):
    """Whether the tokens at positions i (a tensor) are the last of their grid row."""
    if c["grid_w"] == 0:
        return torch.zeros_like(i, dtype=torch.bool)
    j = i - c["prefix"]
    return (j >= 0) & ((j + 1) % c["grid_w"] == 0)


def _linear_recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, h_{-1} = 0, by doubling: after step n every entry
    spans 2^n tokens."""
    n = 1
    while n < a.shape[1]:
        b = torch.cat((b[:, :n], b[:, n:] + a[:, n:] * b[:, :-n]), dim=1)
        a = torch.cat((a[:, :n], a[:, n:] * a[:, :-n]), dim=1)
        n *= 2
    return b


def _plain_scan(s, c, mode):
    dt = s["x"].dtype
    x, z = s["x"].float(), s["gate"].float()
    lam = torch.sigmoid(z) if c["logits"] else z
    rest = torch.sigmoid(-z) if c["logits"] else 1 - z
    gain = rest if c["tied"] else torch.ones_like(rest)
    if mode == "step":
        a = torch.where(_ends_row(s["pos"], c)[:, None], torch.ones_like(lam), lam)
        h = a * s["h_in"] + gain * x
        return dict(y=h.to(dt), h=h)
    ends = _ends_row(torch.arange(x.shape[1], device=x.device), c)[None, :, None]
    a = torch.where(ends, torch.ones_like(lam), lam)
    b = gain * x
    b[:, 0] += a[:, 0] * s["h_in"]
    h = _linear_recurrence(a, b)
    out = dict(y=h.to(dt), h=h[:, -1].clone())
    if mode == "forward":
        return out
    # g_t = dy_t + a_{t+1} g_{t+1}, the same recurrence from the end
    dy = s["dy"].to(torch.float32, copy=True)
    dy[:, -1] += s["dh_out"]
    after = torch.cat((torch.zeros_like(a[:, :1]), a[:, 1:].flip(1)), dim=1)
    g = _linear_recurrence(after, dy.flip(1)).flip(1)
    before = torch.cat((s["h_in"][:, None], h[:, :-1]), dim=1)
    dlam = torch.where(ends, torch.zeros_like(g), g * before)
    if c["tied"]:
        dlam = dlam - g * x
    if c["logits"]:
        dlam = dlam * lam * rest
    out.update(dx=(gain * g).to(dt), dgate=dlam.to(dt), dh_in=a[:, 0] * g[:, 0])
    return out


def _rotation(s, c, T, dev):
    """cos and sin [B or 1, T, 1, d/2] of every token's pairs; tokens before the grid are not turned."""
    pos = s["pos"].long()[:, None] if "pos" in s else torch.zeros(1, 1, dtype=torch.long, device=dev)
    i = pos + torch.arange(T, device=dev)[None, :]
    if c["grid_w"] == 0:
        t = s["table"][i]
    else:
        j = (i - c["prefix"]).clamp(min=0)
        t = torch.cat((s["table"][j // c["grid_w"]], s["table"][j % c["grid_w"]]), dim=2)
        still = torch.tensor([1.0, 0.0], device=dev)
        t = torch.where((i >= c["prefix"])[:, :, None, None], t, still)
    return t[..., 0].unsqueeze(2), t[..., 1].unsqueeze(2)


def _turn(x, cos, sin, half):
    n = x.shape[-1] // 2
    x0, x1 = (x[..., :n], x[..., n:]) if half else (x[..., 0::2], x[..., 1::2])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    return torch.cat((y0, y1), dim=-1) if half else torch.stack((y0, y1), dim=-1).flatten(-2)


def _plain_rope_one(x, w, cos, sin, half, dy=None):
    r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + 1e-6)
    if dy is None:
        return _turn(x * r * w, cos, sin, half)
    u = _turn(dy, cos, -sin, half)
    xn = x * r
    uw = u * w
    return r * (uw - xn * (uw * xn).mean(dim=-1, keepdim=True)), (u * xn).sum(dim=(0, 1, 2))


def _plain_rope(s, c, mode):
    dt = s["q"].dtype
    cos, sin = _rotation(s, c, s["q"].shape[1], s["q"].device)
    q, k = s["q"].float(), s["k"].float()
    out = dict(q=_plain_rope_one(q, s["wq"], cos, sin, c["half"]).to(dt),
               k=_plain_rope_one(k, s["wk"], cos, sin, c["half"]).to(dt))
    if mode == "train":
        dq, dwq = _plain_rope_one(q, s["wq"], cos, sin, c["half"], s["dq_out"].float())
        dk, dwk = _plain_rope_one(k, s["wk"], cos, sin, c["half"], s["dk_out"].float())
        out.update(dq=dq.to(dt), dk=dk.to(dt), dwq=dwq, dwk=dwk)
    return out


def _softmax(x):
    """Row softmax of masked scores (-inf where masked): (p, log of the sum); an empty row gives 0, -inf."""
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    n = p.sum(dim=-1, keepdim=True)
    return p / torch.where(n == 0, torch.ones_like(n), n), (m + torch.log(n)).squeeze(-1)


def _plain_window_step(s, c):
    B, Hk, d = s["k"].shape
    G = c["Hq"] // Hk
    W, S = c["window"], c["sinks"]
    pos = s["pos"].long()
    slot = torch.where(pos < S, pos, S + (pos - S) % W)
    live = pos >= 0
    rows, slot = torch.arange(B, device=pos.device), slot.clamp(min=0)
    for_k = torch.where(live[:, None, None], s["k"], s["k_cache"][rows, slot])
    for_v = torch.where(live[:, None, None], s["v"], s["v_cache"][rows, slot])
    s["k_cache"][rows, slot] = for_k
    s["v_cache"][rows, slot] = for_v
    k, v = s["k_cache"].float(), s["v_cache"].float()                         # [B, slots, Hk, d]
    q = s["q"].float().view(B, Hk, G, d)
    n = torch.arange(S + W, device=pos.device)
    seen = torch.where(n < S, n <= pos[:, None], n - S < (pos[:, None] + 1 - S))  # filled so far
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
    p, _ = _softmax(torch.where(seen[:, None, None, :], x, torch.full_like(x, -math.inf)))
    o = torch.matmul(p, v.permute(0, 2, 1, 3)).view(B, c["Hq"], d).to(s["q"].dtype)
    return dict(o=o, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_window(s, c, mode):
    if mode == "step":
        return _plain_window_step(s, c)
    dt = s["q"].dtype
    B, T, Hk, d = s["k"].shape
    Hq = c["Hq"]
    G = Hq // Hk
    rows = lambda x: x.float().view(B, T, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * T, d)   # noqa: E731
    back = lambda x: x.view(B, Hk, G, T, d).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, d).to(dt)        # noqa: E731
    q, k, v = rows(s["q"]), s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2)
    t = torch.arange(T, device=q.device)
    seen = (t[None, :] <= t[:, None]) & ((t[None, :] > t[:, None] - c["window"]) | (t[None, :] < c["sinks"]))
    if "lengths" in s:
        inside = t[None, :] < s["lengths"][:, None]
        seen = seen & inside[:, :, None] & inside[:, None, :]
    seen = seen.view(-1, 1, 1, T, T)
    scale = 1 / math.sqrt(d)
    x = (torch.matmul(q, k.transpose(2, 3)) * scale).view(B, Hk, G, T, T)
    p, lse = _softmax(x.masked_fill_(~seen, -math.inf))
    p = p.view(B, Hk, G * T, T)
    o = torch.matmul(p, v)
    out = dict(o=back(o), lse=lse.reshape(B, Hq, T))
    if mode == "forward":
        return out
    do = rows(s["do"])
    dv = torch.matmul(p.transpose(2, 3), do)
    dp = torch.matmul(do, v.transpose(2, 3))
    ds = p * (dp - (do * o).sum(dim=-1, keepdim=True)) * scale
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    out.update(dq=back(dq), dk=dk.transpose(1, 2).to(dt), dv=dv.transpose(1, 2).to(dt))
    return out


_PLAIN = dict(scan=_plain_scan, rope=_plain_rope, window=_plain_window)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def _pairs(n, window, sinks):
    """Visible (query, key) pairs of a sequence of n tokens."""
    total = 0
    for t in range(n):
        low = max(0, t - window + 1)
        total += t + 1 - low + min(sinks, low)
    return total


def work(case):
    e = 2 if case["dtype"] == _BF16 else 4
    B, T = case["B"], case["T"]
    train = case["mode"] == "train"
    if case["op"] == "scan":
        n, state = B * T * case["C"], B * case["C"] * 4
        # forward: x, gate in, y out; backward: x, gate, dy in, dx, dgate out
        return dict(bytes=n * e * (8 if train else 3) + state * (4 if train else 2), flops=n * (14 if train else 4))
    d, Hq, Hk = case["d"], case["Hq"], case["Hk"]
    if case["op"] == "rope":
        n = B * T * (Hq + Hk) * d
        return dict(bytes=n * e * (5 if train else 2), flops=n * (16 if train else 6))
    if case["mode"] == "step":
        slots = sum(min(p + 1, case["window"] + case["sinks"]) for p in _positions(case))
        return dict(bytes=(slots * Hk * 2 + B * Hk * 2 + B * Hq * 2) * d * e, flops=4 * slots * Hq * d)
    pairs = sum(_pairs(n, case["window"], case["sinks"]) for n in (_lengths(case) or [T] * B))
    q, k = B * T * Hq * d * e, B * T * Hk * d * e
    lse = B * T * Hq * 4
    # forward: q, k, v in, o out; training adds q, k, v, o, do in and dq, dk, dv out
    return dict(bytes=(2 * q + 2 * k + lse) + ((4 * q + 4 * k + lse) if train else 0),
                flops=pairs * Hq * d * (14 if train else 4))


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return dict(scan=_exact_scan, rope=_exact_rope, window=_exact_window)[case["op"]](s, case)


def _exact_scan(s, c):
    x, z = s["x"].double(), s["gate"].double()
    f = 1 / (1 + torch.exp(-z)) if c["logits"] else z
    r = 1 / (1 + torch.exp(z)) if c["logits"] else 1 - z
    u = r * x if c["tied"] else x

    def last_of_row(i):
        return c["grid_w"] > 0 and i >= c["prefix"] and (i - c["prefix"] + 1) % c["grid_w"] == 0

    h = s["h_in"].double()
    if c["mode"] == "step":
        whole = torch.tensor([last_of_row(i) for i in _positions(c)], device=h.device)
        h = f.masked_fill(whole[:, None], 1.0) * h + u
        return dict(y=h, h=h)
    T = x.shape[1]
    y = torch.empty_like(x)
    for t in range(T):
        h = (h if last_of_row(t) else f[:, t] * h).add(u[:, t])
        y[:, t] = h
    if c["mode"] == "forward":
        return dict(y=y, h=y[:, -1])
    dx, dz = torch.empty_like(x), torch.empty_like(x)
    carry = s["dh_out"].double()
    for t in range(T - 1, -1, -1):
        g = carry + s["dy"][:, t].double()
        prev = y[:, t - 1] if t else s["h_in"].double()
        df = torch.zeros_like(g) if last_of_row(t) else g * prev
        if c["tied"]:
            df = df - g * x[:, t]
        dz[:, t] = df * (f[:, t] * r[:, t]) if c["logits"] else df
        dx[:, t] = g * r[:, t] if c["tied"] else g
        carry = g if last_of_row(t) else g * f[:, t]
    return dict(y=y, h=y[:, -1], dx=dx, dgate=dz, dh_in=carry)


def _exact_rope(s, c):
    dev = s["q"].device
    T, n = c["T"], c["d"] // 2
    start = torch.tensor(_spread(c["B"], 0, 256) if c["ragged"] else [0], device=dev)
    i = (start[:, None] + torch.arange(T, device=dev)).double()
    if c["grid_w"]:
        freq = 10000.0 ** (-torch.arange(n // 2, device=dev).double() / (n // 2))
        j = i - c["prefix"]
        row = torch.floor(j / c["grid_w"])
        col = j - row * c["grid_w"]
        angle = torch.cat((row[..., None] * freq, col[..., None] * freq), -1) * (j >= 0)[..., None]
    else:
        angle = i[..., None] * 10000.0 ** (-torch.arange(n, device=dev).double() / n)
    # a pair as one complex number
    spin = torch.polar(torch.ones_like(angle), angle)[:, :, None]
    to_c = (lambda v: torch.complex(v[..., :n], v[..., n:])) if c["half"] else (
        lambda v: torch.view_as_complex(v.unflatten(-1, (n, 2)).contiguous()))
    to_r = (lambda v: torch.cat((v.real, v.imag), -1)) if c["half"] else (lambda v: torch.view_as_real(v).flatten(-2))
    out = {}
    for name, w in (("q", s["wq"].double()), ("k", s["wk"].double())):
        x = s[name].double()
        size = torch.sqrt((x * x).sum(-1, keepdim=True) / c["d"] + 1e-6)
        out[name] = to_r(to_c(w * x / size) * spin)
        if c["mode"] == "train":
            dw = to_r(to_c(s["d%s_out" % name].double()) * spin.conj())
            dn = dw * w
            out["dw" + name] = (dw * x / size).sum((0, 1, 2))
            out["d" + name] = dn / size - x * (dn * x).sum(-1, keepdim=True) / (c["d"] * size ** 3)
    return out


def _exact_window(s, c):
    W, S, d = c["window"], c["sinks"], c["d"]
    G = c["Hq"] // c["Hk"]
    f = 1 / math.sqrt(d)
    if c["mode"] == "step":
        o = torch.zeros_like(s["q"], dtype=torch.float64)
        kc, vc = s["k_cache"].clone(), s["v_cache"].clone()
        for b, p in enumerate(_positions(c)):
            if p < 0:
                continue
            at = p if p < S else S + (p - S) % W
            kc[b, at], vc[b, at] = s["k"][b], s["v"][b]
            n = min(p + 1, S + W)
            k, v = (m[b, :n].double().repeat_interleave(G, dim=1) for m in (kc, vc))
            a = torch.softmax(torch.einsum("hd,nhd->hn", s["q"][b].double(), k) * f, -1)
            o[b] = torch.einsum("hn,nhd->hd", a, v)
        return dict(o=o, k_cache=kc.double(), v_cache=vc.double())
    B, T = c["B"], c["T"]
    train = c["mode"] == "train"
    q64 = lambda n: torch.zeros_like(s[n], dtype=torch.float64)   # noqa: E731
    out = dict(o=q64("q"), lse=torch.full((B, c["Hq"], T), -math.inf, dtype=torch.float64, device=s["q"].device))
    if train:
        out.update(dq=q64("q"), dk=q64("k"), dv=q64("k"))
    lengths = _lengths(c) or [T] * B
    size = max(1, (1 << 24) // T)                                  # rows at a time
    for b, n in enumerate(lengths):
        for h in range(c["Hq"]):
            k, v = s["k"][b, :n, h // G].double(), s["v"][b, :n, h // G].double()
            for t0 in range(0, n, size):
                t = torch.arange(t0, min(n, t0 + size), device=k.device)[:, None]
                u = torch.arange(n, device=k.device)[None, :]
                hidden = (u > t) | ((u <= t - W) & (u >= S))
                q = s["q"][b, t0:t0 + size, h][: t.shape[0]].double()
                x = (q @ k.T * f).masked_fill(hidden, -math.inf)
                z = torch.logsumexp(x, -1)
                a = torch.exp(x - z[:, None])
                o = a @ v
                at = slice(t0, t0 + t.shape[0])
                out["o"][b, at, h], out["lse"][b, h, at] = o, z
                if train:
                    g = s["do"][b, at, h].double()
                    da = g @ v.T
                    dx = a * (da - (a * da).sum(-1, keepdim=True)) * f
                    out["dq"][b, at, h] = dx @ k
                    out["dk"][b, :n, h // G] += dx.T @ q
                    out["dv"][b, :n, h // G] += a.T @ g
    return out
