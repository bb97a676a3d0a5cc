"""Plain float64 forms of the operators beside LASAD, on the CPU, written from their formulas.

The gradients are torch autograd's of these forms.  ``window_bounds`` adds how far a call may be off
that rounds its weights and score gradients to bf16 where they enter a product."""
import math

import torch


def ends_row(i, grid_w, prefix):
    return grid_w > 0 and i >= prefix and (i - prefix + 1) % grid_w == 0


def scan(x, gate, h_in=None, grid_w=0, prefix=0, t0=0, tied=True, logits=False):
    """(y, h_out) of x, gate [B,T,C] in float64."""
    lam = torch.sigmoid(gate) if logits else gate
    rest = torch.sigmoid(-gate) if logits else 1 - gate
    h = torch.zeros_like(x[:, 0]) if h_in is None else h_in
    ys = []
    for t in range(x.shape[1]):
        a = torch.ones_like(h) if ends_row(t0 + t, grid_w, prefix) else lam[:, t]
        h = a * h + (rest[:, t] * x[:, t] if tied else x[:, t])
        ys.append(h)
    return torch.stack(ys, 1), h


def rope_one(x, w, pos, grid_w, prefix, half, eps, base=10000.0):
    """x [B,T,H,d] float64, pos [B] or an int: the first token's position."""
    B, T, H, d = x.shape
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w
    n = d // 2
    start = torch.as_tensor(pos).reshape(-1, 1).expand(B, 1)
    i = start + torch.arange(T)
    ang = torch.zeros(B, T, n, dtype=torch.float64)
    for m in range(n):
        if grid_w == 0:
            ang[:, :, m] = i.double() * base ** (-m / n)
        else:
            j = i - prefix
            k = torch.div(j, grid_w, rounding_mode="floor") if m < n // 2 else j % grid_w
            ang[:, :, m] = torch.where(j >= 0, k.double() * base ** (-(m % (n // 2)) / (n // 2)), torch.zeros(()).double())
    c, s = ang.cos()[:, :, None], ang.sin()[:, :, None]
    if half:
        a, b = y[..., :n], y[..., n:]
        return torch.cat((a * c - b * s, a * s + b * c), -1)
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)


def seen(T, window, sinks, n):
    t = torch.arange(T)
    d = t[:, None] - t[None, :]
    return (d >= 0) & ((d < window) | (t[None, :] < sinks)) & (t[:, None] < n) & (t[None, :] < n)


def window(q, k, v, win, sinks=0, scale=None, lengths=None):
    """(o, lse) of q [B,T,Hq,d], k, v [B,T,Hk,d] in float64; what lies past a sequence's end is not used."""
    B, T, Hq, d = q.shape
    G = Hq // k.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    o, lse = torch.zeros_like(q), torch.full((B, Hq, T), -math.inf, dtype=torch.float64)
    os = []
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        mask = seen(T, win, sinks, n)[:n, :n]
        qb = q[b, :n].transpose(0, 1)
        kb, vb = (x[b, :n].transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
        s = (qb @ kb.transpose(1, 2) * scale).masked_fill(~mask, -math.inf)
        if n:
            lse[b, :, :n] = torch.logsumexp(s, -1).detach()
            ob = (torch.softmax(s, -1) @ vb).transpose(0, 1)
        else:
            ob = q.new_zeros(0, Hq, d)
        os.append(torch.cat((ob, ob.new_zeros(T - n, Hq, d))))
    return torch.stack(os), lse


def window_bounds(q, k, v, do, win, sinks=0, scale=None, lengths=None, u=2.0 ** -8, acc=2.0 ** -20):
    """Error bounds {o, dq, dk, dv} of a call whose tensors, p and ds carry a relative error of u and
    whose sums, statistics and exponentials one of acc of the sum of magnitudes."""
    B, T, Hq, d = q.shape
    Hk = k.shape[2]
    G = Hq // Hk
    scale = 1 / math.sqrt(d) if scale is None else scale
    size = abs(scale)
    out = {n: torch.zeros_like(x) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", k))}
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        mask = seen(T, win, sinks, n)[:n, :n]
        for h in range(Hq):
            qh, gh, kh, vh = q[b, :n, h], do[b, :n, h], k[b, :n, h // G], v[b, :n, h // G]
            if n == 0:
                continue
            x = (qh @ kh.T * scale).masked_fill(~mask, -math.inf)
            p = torch.softmax(x, -1)
            # an error of the exponent is one of p: acc of the sum of magnitudes of q.k and of the statistics
            e = u + acc * (2 + (qh.abs() @ kh.abs().T * size) + x.abs().masked_fill(~mask, 0).amax(-1, keepdim=True))
            pe = p * e
            o = p @ vh
            oerr = pe @ vh.abs() + u * o.abs()
            out["o"][b, :n, h] = oerr
            dp = gh @ vh.T
            delta = (gh * o).sum(-1, keepdim=True)
            derr = (gh.abs() * oerr).sum(-1, keepdim=True) + acc * (gh.abs() * o.abs()).sum(-1, keepdim=True)
            ds = p * (dp - delta) * scale
            dserr = pe * (dp - delta).abs() * size + p * size * (derr + acc * (gh.abs() @ vh.abs().T)) + u * ds.abs()
            out["dq"][b, :n, h] = dserr @ kh.abs() + u * (ds @ kh).abs() + acc * (ds.abs() @ kh.abs())
            out["dk"][b, :n, h // G] += dserr.T @ qh.abs() + (u + acc) * (ds.abs().T @ qh.abs())
            out["dv"][b, :n, h // G] += pe.T @ gh.abs() + (u + acc) * (p.T @ gh.abs())
    return out


def window_step(q, k, v, k_cache, v_cache, pos, win, sinks=0, scale=None):
    """(o, k_cache, v_cache) after the step, float64; the caches come back as copies."""
    B, Hq, d = q.shape
    G = Hq // k.shape[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    kc, vc, o = k_cache.clone(), v_cache.clone(), torch.zeros_like(q)
    for b in range(B):
        p = int(pos[b])
        if p < 0:
            continue
        slot = p if p < sinks else sinks + (p - sinks) % win
        kc[b, slot], vc[b, slot] = k[b], v[b]
        tokens = [s for s in range(p + 1) if p - s < win or s < sinks]
        slots = [s if s < sinks else sinks + (s - sinks) % win for s in tokens]
        assert len(set(slots)) == len(slots)
        for h in range(Hq):
            a = torch.softmax(kc[b, slots, h // G] @ q[b, h] * scale, 0)
            o[b, h] = a @ vc[b, slots, h // G]
    return o, kc, vc
