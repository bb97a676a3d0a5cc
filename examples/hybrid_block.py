#!/usr/bin/env python
"""A small hybrid stack over a raster-flattened grid: every block mixes tokens three ways, side by side
on the same [B,T,H,d] tensors, and all three know the grid --

    LASAD           linear attention with spatial decay (carried as a state of d x d per head),
    window          softmax attention over the last tokens and the first ones, queries and keys normed
                    and turned by their row and column (carried as a ring cache),
    recurrence      h <- lambda h + (1 - lambda) x per channel (carried as one number per channel).

    python examples/hybrid_block.py [train] [generate]

``train`` fits the window and the recurrence branches (the framework has no gradient of LASAD) to a
random teacher for a few steps, through torch.autograd.  ``generate`` runs a prefix through all three
at once, puts what they carry aside and continues it token by token; it checks that both ways give
the same rows.
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2507_01652_b200 import binding  # noqa: E402


class Scan(torch.autograd.Function):
    """y of the gated linear recurrence over [B,T,C]; z is the gate's pre-activation."""

    @staticmethod
    def forward(fn, ctx, x, z, grid_w):
        y, _, saved = ctx.lasad_scan_forward(x, z, grid_w=grid_w, logits=True, want_state=False, save=True)
        fn.save_for_backward(x, z, saved)
        fn.ctx, fn.grid_w = ctx, grid_w
        return y

    @staticmethod
    def backward(fn, dy):
        x, z, saved = fn.saved_tensors
        dx, dz, _ = fn.ctx.lasad_scan_backward(x, z, saved, dy.contiguous(), grid_w=fn.grid_w, logits=True, want_state=False)
        return None, dx, dz, None


class NormRope(torch.autograd.Function):
    """Queries and keys normed per head and turned by their place on the grid."""

    @staticmethod
    def forward(fn, ctx, q, k, wq, wk, table, grid_w):
        fn.save_for_backward(q, k, wq, wk, table)
        fn.ctx, fn.grid_w = ctx, grid_w
        return ctx.lasad_qk_norm_rope(q, k, table, wq, wk, grid_w=grid_w)

    @staticmethod
    def backward(fn, dq_out, dk_out):
        q, k, wq, wk, table = fn.saved_tensors
        dq, dk, dwq, dwk = fn.ctx.lasad_qk_norm_rope_backward(q, k, table, dq_out.contiguous(), dk_out.contiguous(), wq, wk,
                                                              grid_w=fn.grid_w)
        return None, dq, dk, dwq, dwk, None, None


class Window(torch.autograd.Function):
    """Softmax attention over the last `window` tokens and the first `sinks`."""

    @staticmethod
    def forward(fn, ctx, q, k, v, window, sinks):
        o, lse = ctx.lasad_window_attention(q, k, v, window, sinks, want_lse=True)
        fn.save_for_backward(q, k, v, o, lse)
        fn.ctx, fn.window, fn.sinks = ctx, window, sinks
        return o

    @staticmethod
    def backward(fn, do):
        dq, dk, dv = fn.ctx.lasad_window_attention_backward(*fn.saved_tensors, do.contiguous(), fn.window, fn.sinks)
        return None, dq, dk, dv, None, None


class Block:
    """One block: projections in bf16, three mixers, their sum projected back."""

    def __init__(self, ctx, width=256, heads=4, key_heads=2, grid_w=16, rows=16, window=32, sinks=1, seed=0):
        gen = torch.Generator().manual_seed(seed)
        d = width // heads
        kv = key_heads * d

        def w(i, o):
            return (torch.randn(i, o, generator=gen) / i ** 0.5).bfloat16().cuda().requires_grad_()
        self.ctx, self.d, self.heads, self.key_heads = ctx, d, heads, key_heads
        self.grid_w, self.window, self.sinks, self.cuts = grid_w, window, sinks, (width, kv, kv, width, width)
        self.into, self.out = w(width, sum(self.cuts)), w(width, width)
        self.wq, self.wk = (torch.ones(d, device="cuda").requires_grad_() for _ in range(2))
        self.decay = torch.linspace(0.9, 0.99, heads, device="cuda")
        self.table = binding.rope_table(max(rows, grid_w), d, True, device="cuda")

    def parameters(self):
        return [self.into, self.out, self.wq, self.wk]

    def project(self, u):
        """q, k, v as heads; x and the gate's pre-activation of the recurrence as channels."""
        q, k, v, x, z = (u @ self.into).split(self.cuts, -1)
        lead = u.shape[:-1]
        return (q.view(*lead, self.heads, self.d), k.view(*lead, self.key_heads, self.d), v.view(*lead, self.key_heads, self.d),
                x, z)

    def shared(self, k):
        """Every query head's key head, for LASAD, which has as many of one as of the other."""
        return k.repeat_interleave(self.heads // self.key_heads, -2)

    def train(self, u):
        """The window and the recurrence branches; differentiable."""
        q, k, v, x, z = self.project(u)
        a, b = NormRope.apply(self.ctx, q, k, self.wq, self.wk, self.table, self.grid_w)
        o = Window.apply(self.ctx, a, b, v, self.window, self.sinks)
        return (o.flatten(-2) + Scan.apply(self.ctx, x, z, self.grid_w)) @ self.out

    def prefill(self, u):
        """All three over u [B,T,width]; returns the rows and what the next token needs."""
        q, k, v, x, z = self.project(u)
        a, b = self.ctx.lasad_qk_norm_rope(q, k, self.table, self.wq, self.wk, grid_w=self.grid_w)
        o, _ = self.ctx.lasad_window_attention(a, b, v, self.window, self.sinks)
        y, h, _ = self.ctx.lasad_scan_forward(x, z, grid_w=self.grid_w, logits=True)
        s, state = self.ctx.lasad_forward(a, self.shared(b), self.shared(v), self.decay, self.grid_w)
        caches = [b.new_empty(u.shape[0], self.sinks + self.window, self.key_heads, self.d) for _ in range(2)]
        self.ctx.lasad_window_cache_store(b, v, *caches, self.window, self.sinks)
        return (o.flatten(-2) + y + s.flatten(-2)) @ self.out, (state, h, *caches)

    def step(self, u, carried, pos):
        """One token u [B,width] at the positions pos int32 [B]; what is carried is updated in place."""
        state, h, kc, vc = carried
        q, k, v, x, z = self.project(u)
        a, b = self.ctx.lasad_qk_norm_rope(q[:, None], k[:, None], self.table, self.wq, self.wk, grid_w=self.grid_w, pos=pos)
        a, b = a[:, 0], b[:, 0]
        o = self.ctx.lasad_window_attention_step(a, b, v, kc, vc, pos, self.window, self.sinks)
        y, _ = self.ctx.lasad_scan_step(x, z, h, grid_w=self.grid_w, pos=pos, logits=True)
        s = self.ctx.lasad_decode_step_pos(a, self.shared(b), self.shared(v), self.decay, state, pos, grid_w=self.grid_w)
        return (o.flatten(-2) + y + s.flatten(-2)) @ self.out


def train(steps=20, B=2, T=256, width=256):
    """Losses of a few steps of plain gradient descent towards a random teacher."""
    ctx = binding.Lasad(torch.cuda.current_device())
    student, teacher = Block(ctx, width, seed=1), Block(ctx, width, seed=2)
    u = torch.randn(B, T, width, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    with torch.no_grad():
        goal = teacher.train(u).float()
    losses = []
    for _ in range(steps):
        loss = (student.train(u).float() - goal).square().mean()
        grads = torch.autograd.grad(loss, student.parameters())
        with torch.no_grad():
            for p, g in zip(student.parameters(), grads):
                p -= (20.0 if p.dim() > 1 else 1.0) * g.to(p.dtype)
        losses.append(loss.item())
    assert ctx.device_status() == 0
    ctx.close()
    return losses


@torch.no_grad()
def generate(B=3, T=200, prefix=70, width=256):
    """Largest difference between the rows of one pass and those of a prefix continued token by
    token, as a part of the largest row."""
    ctx = binding.Lasad(torch.cuda.current_device())
    block = Block(ctx, width)
    u = torch.randn(B, T, width, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    whole, _ = block.prefill(u)
    _, carried = block.prefill(u[:, :prefix])
    worst = 0.0
    for t in range(prefix, T):
        row = block.step(u[:, t], carried, torch.full((B,), t, dtype=torch.int32, device="cuda"))
        worst = max(worst, float((row.float() - whole[:, t].float()).abs().max()))
    assert ctx.device_status() == 0
    ctx.close()
    return worst / float(whole.float().abs().max())


if __name__ == "__main__":
    what = sys.argv[1:] or ["train", "generate"]
    if "train" in what:
        losses = train()
        print(f"train: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    if "generate" in what:
        print(f"generate: token by token against one pass: {generate():.2e} of the largest value")
