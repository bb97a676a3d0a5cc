"""Packed attention where the running maximum of a row moves: P of the tile is formed again, and O and the sum are
scaled.  With scores of ordinary size that is rare after a sequence's first tile, so these make it happen."""
import math

import pytest
import torch

from tests import _sequences_ref as ref
from tests.test_gpu_mixers import BF16, F32, ctx, d64, gen, near, rnd  # noqa: F401
from tests.test_gpu_sequences import both_ways, inside

pytestmark = pytest.mark.gpu


def growing(T, heads, seed, step=14.0):
    """Keys whose score grows by ``step`` (in log2) or a little more from one tile of 64 to the next, for every query."""
    g = gen(seed)
    q, k = rnd(g, T, heads, 64, std=0.5, dtype=BF16), rnd(g, T, heads, 64, std=0.5, dtype=BF16)
    q[:, :, 0] = 8.0
    # scale log2(e) q.k = 0.125 x 1.4427 x 8 k_0
    k[:, :, 0] = ((torch.arange(T) // 64).float() * (step / (0.125 * 1.4427 * 8.0)))[:, None].to(BF16)
    return q, k, rnd(g, T, heads, 64, dtype=BF16)


@pytest.mark.parametrize("lengths", [(64 * 9 + 5,), (577, 130, 300)])
def test_a_maximum_that_moves_in_every_tile(ctx, lengths):      # noqa: F811
    """The tile's P with the old maximum, 2^14 and more too large, may not stay where the new one belongs.  Every one of
    40 launches is the formula's, and has the first one's bits."""
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    q, k, v = growing(offsets[-1], 3, 21)
    want, want_lse = ref.packed(d64(q), d64(k), d64(v), offsets)
    bound = ref.packed_bounds(d64(q), d64(k), d64(v), torch.zeros_like(want), offsets)["o"]
    at = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    dev = [t.cuda() for t in (q, k, v)]
    outs = [ctx.lasad_packed_attention(*dev, at, want_lse=True) for _ in range(40)]
    assert ctx.device_status() == 0
    inside("o", outs[0][0], want, bound)
    near(outs[0][1], want_lse, F32, "lse", extra=2.0 ** -18)
    for o, lse in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(lse, outs[0][1])


def test_every_launch_of_many_has_the_same_bits(ctx):      # noqa: F811
    """Forward and gradient back to back, ordinary scores and growing ones: each launch against the first."""
    g = gen(22)
    T = 1300
    at = torch.tensor([0, 700, 701, T], dtype=torch.int32, device="cuda")
    for q, k, v in ((rnd(g, T, 4, 64, std=1.5, dtype=BF16), rnd(g, T, 4, 64, dtype=BF16), rnd(g, T, 4, 64, dtype=BF16)), growing(T, 4, 23)):
        q, k, v, do = (t.cuda() for t in (q, k, v, rnd(g, T, 4, 64, dtype=BF16)))
        first, same = None, torch.ones((), dtype=torch.bool, device="cuda")
        for _ in range(30):
            o, lse = ctx.lasad_packed_attention(q, k, v, at, want_lse=True)
            got = (o, lse) + ctx.lasad_packed_attention_backward(q, k, v, o, lse, do, at)
            first = first or got
            for a, b in zip(first, got):
                same &= (a == b).all()
        assert bool(same) and ctx.device_status() == 0


def unseen(seed, first):
    """Two sequences of keys and queries: row 200 of the first (with 31 others in its warp) has scores of -infinity, by
    overflow, with the keys before ``first``; the other rows do not see that channel of the keys.  Row 203's scores grow
    by about 40 (in log2) with key 70, of the second tile."""
    g = gen(seed)
    n, T = 320, 420
    q, k, v = (rnd(g, T, h, 64, std=0.5, dtype=BF16) for h in (2, 1, 1))
    q[:, :, :2] = 0.0
    k[:, :, :2] = 0.0
    k[:first, :, 0] = -1e30
    q[200, :, 0] = 1e30
    k[70, :, 1], q[203, :, 1] = 16.0, 14.0
    do = rnd(g, T, 2, 64, dtype=BF16)
    return [q, k, v, do], [0, n, T]


@pytest.mark.parametrize("first", [128, 201])
def test_a_row_that_has_seen_nothing_beside_one_that_grows(ctx, first):      # noqa: F811
    """Scores that overflow are -infinity, and weigh nothing: row 200's output is that of the keys it does see, and 0 with
    lse -infinity where there are none, whatever its neighbours do and on both implementations."""
    (q, k, v, do), offsets = unseen(31, first)
    at = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    seen = k.clone()
    seen[:, :, 0] = 0.0
    other = q.clone()
    other[200, :, 0] = 0.0
    want, want_lse = ref.packed(d64(other), d64(seen), d64(v), offsets)
    bounds = ref.packed_bounds(d64(other), d64(seen), d64(v), d64(do), offsets)
    n = 201 - first
    if n:                                         # row 200 as the last row of a sequence of the keys that it sees
        part = [d64(t)[first:201] for t in (other, seen, v, do)]
        o, lse = ref.packed(*part[:3], [0, n])
        want[200], want_lse[:, 200] = o[-1], lse[:, -1]
        bounds["o"][200] = ref.packed_bounds(*part, [0, n])["o"][-1]
    else:
        want[200], want_lse[:, 200], bounds["o"][200] = 0.0, -math.inf, 0.0
    for way in both_ways(ctx, [t.cuda() for t in (q, k, v, do)], at):
        inside("o", way[0], want, bounds["o"])
        near(way[1], want_lse, F32, "lse", extra=2.0 ** -18)


@pytest.mark.parametrize("n", [513, 577, 70])
def test_rows_behind_a_sequence_do_not_move_its_maximum(ctx, n):      # noqa: F811
    """A warp's last rows may belong to another sequence or to none.  Theirs have scores of hundreds here, so their
    maxima move in tile after tile; the sequence's own rows get the bits that they get alone."""
    g = gen(41)
    T = 800
    q, k, v = (rnd(g, T, h, 64, std=s, dtype=BF16) for h, s in ((4, 1.5), (2, 1.0), (2, 1.0)))
    q[n:] *= 60.0
    dev = [t.cuda() for t in (q, k, v)]
    alone = ctx.lasad_packed_attention(*[t[:n].contiguous() for t in dev], torch.tensor([0, n], dtype=torch.int32, device="cuda"), want_lse=True)
    for offsets in ([0, n, T], [0, n]):
        o, lse = ctx.lasad_packed_attention(*dev, torch.tensor(offsets, dtype=torch.int32, device="cuda"), want_lse=True)
        assert torch.equal(o[:n], alone[0]) and torch.equal(lse[:, :n], alone[1])
    assert ctx.device_status() == 0


def test_the_gradient_of_a_row_that_has_seen_nothing(ctx):      # noqa: F811
    """Such a row is empty (o 0, lse -infinity): its gradient is 0, and nothing of it comes to its keys and values."""
    (q, k, v, do), offsets = unseen(32, 201)
    at = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    leaves = [d64(t) for t in (q, k, v)]
    leaves[0][200, :, 0] = 0.0
    leaves[1][:, :, 0] = 0.0
    leaves = [t.requires_grad_() for t in leaves]
    without = do.clone()
    without[200] = 0.0                            # (then nothing comes from the row)
    want = torch.autograd.grad(ref.packed(*leaves, offsets)[0], leaves, d64(without))
    bounds = ref.packed_bounds(*[t.detach() for t in leaves], d64(without), offsets)
    for way in both_ways(ctx, [t.cuda() for t in (q, k, v, do)], at):
        assert bool((way[2][200] == 0).all())
        for name, got, w in zip(("dq", "dk", "dv"), way[2:], want):
            got, w, b = got.clone(), w.clone(), bounds[name]
            if name == "dq":
                got[:, :, 0], w[:, :, 0] = 0.0, 0.0      # (dq_0 is ds k_0, ...)
            inside(name, got, w, b)
