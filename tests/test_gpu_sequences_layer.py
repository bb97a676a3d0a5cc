"""A layer that attends to whole sequences with the framework's own norm and rotation: a pack goes through
``lasad_qk_norm_rope`` as one row of one token for each of its tokens, each with its position.  Every stage is
compared with its formula on what the stage before has given."""
import math

import pytest
import torch

from paper_2507_01652_b200 import binding
from tests import _mixers_ref as mixers
from tests import _sequences_ref as ref
from tests.test_gpu_mixers import BF16, F32, ctx, d64, gen, near, rnd  # noqa: F401
from tests.test_gpu_sequences import cache_of, inside, same_cache, to_64, to_dev

pytestmark = pytest.mark.gpu

LENGTHS, HQ, HK, D, W, PREFIX, EPS = (33, 0, 150, 1), 4, 2, 64, 12, 1, 1e-6
OFFSETS = [0, 33, 33, 183, 184]


def pack(dtype, seed):
    g, n = gen(seed), OFFSETS[-1]
    q, k, v = (rnd(g, n, h, D, dtype=dtype) for h in (HQ, HK, HK))
    weights = [rnd(g, D, mean=1.0, std=0.2) for _ in range(2)]
    pos = torch.cat([torch.arange(m) for m in LENGTHS]).int()
    return g, (q, k, v), weights, pos


def turn(ctx, q, k, weights, pos):      # noqa: F811
    """[N,H,d] at positions pos [N]."""
    table = binding.rope_table(64, D, True, device="cuda")
    kw = dict(q_weight=weights[0].cuda(), k_weight=weights[1].cuda(), grid_w=W, prefix_len=PREFIX, pos=pos.cuda(), eps=EPS)
    a, b = ctx.lasad_qk_norm_rope(q.cuda()[:, None], k.cuda()[:, None], table, **kw)
    return a, b, table, kw


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_training_step_of_the_layer(ctx, dtype):      # noqa: F811
    g, (q, k, v), weights, pos = pack(dtype, 51)
    do = rnd(g, OFFSETS[-1], HQ, D, dtype=dtype)
    qt, kt, table, kw = turn(ctx, q, k, weights, pos)
    leaves = [d64(t).requires_grad_() for t in (q, k, *weights)]
    forms = [mixers.rope_one(x[:, None], w, pos.long(), W, PREFIX, False, EPS) for x, w in zip(leaves[:2], leaves[2:])]
    near(qt, forms[0].detach(), dtype, "q")
    near(kt, forms[1].detach(), dtype, "k")
    at = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
    o, lse = ctx.lasad_packed_attention(qt[:, 0], kt[:, 0], v.cuda(), at, want_lse=True)
    grads = ctx.lasad_packed_attention_backward(qt[:, 0], kt[:, 0], v.cuda(), o, lse, do.cuda(), at)
    inner = [d64(t).requires_grad_() for t in (qt[:, 0], kt[:, 0], v)]
    want = ref.packed(*inner, OFFSETS)[0]
    bounds = ref.packed_bounds(*[t.detach() for t in inner], d64(do), OFFSETS, u=2.0 ** -8 if dtype == BF16 else 2.0 ** -23)
    inside("o", o, want.detach(), bounds["o"])
    for name, got, w in zip(("dq", "dk", "dv"), grads, torch.autograd.grad(want, inner, d64(do))):
        inside(name, got, w, bounds[name])
    back = ctx.lasad_qk_norm_rope_backward(q.cuda()[:, None], k.cuda()[:, None], table, grads[0][:, None], grads[1][:, None], **kw)
    wants = torch.autograd.grad(forms, leaves, [d64(t)[:, None] for t in grads[:2]])
    for name, got, w in zip(("dq", "dk", "dwq", "dwk"), back, wants):
        near(got.view(w.shape), w, F32 if name[1] == "w" else dtype, name, acc=2.0 ** -18 if name[1] == "w" else 2.0 ** -20)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompts_and_tokens_of_the_layer(ctx, dtype):      # noqa: F811
    """Keys that come turned go into the cache without a table, and the same ones through packed attention."""
    g, (q, k, v), weights, pos = pack(dtype, 52)
    B, page, entries = len(LENGTHS), 16, 11
    bt = torch.randperm(B * entries, generator=g).view(B, entries).int()
    cache = cache_of(g, B * entries, HK, page, D)
    dev, want = to_dev(cache), to_64(cache)
    at = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
    qt, kt, _, _ = turn(ctx, q, k, weights, pos)
    o, _ = ctx.lasad_packed_attention(qt[:, 0], kt[:, 0], v.cuda(), at)
    given = [d64(t) for t in (qt[:, 0], kt[:, 0], v)]
    u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -23
    inside("prompts", o, ref.packed(*given, OFFSETS)[0], ref.packed_bounds(*given, torch.zeros_like(given[0]), OFFSETS, u=u)["o"])
    assert ctx.lasad_paged_append(kt[:, 0], v.cuda(), **dev, block_table=bt.cuda(), pos=torch.zeros(B, dtype=torch.int32, device="cuda"),
                                  offsets=at) is None
    ref.append(kt[:, 0].cpu(), v, want, bt, [0] * B, OFFSETS)
    same_cache(dev, want)
    now = list(LENGTHS)
    for _ in range(3):
        q1, k1, v1 = (rnd(g, B, h, D, dtype=dtype) for h in (HQ, HK, HK))
        p = torch.tensor(now, dtype=torch.int32)
        qt, kt, _, _ = turn(ctx, q1, k1, weights, p)
        ctx.lasad_paged_append(kt[:, 0], v1.cuda(), **dev, block_table=bt.cuda(), pos=p.cuda())
        ref.append(kt[:, 0].cpu(), v1, want, bt, now)
        same_cache(dev, want)
        got, lse = ctx.lasad_paged_attention(qt[:, 0], **dev, block_table=bt.cuda(), pos=p.cuda(), want_lse=True)
        o, want_lse, err = ref.paged(d64(qt[:, 0]), want, bt, now, u=2.0 ** -11 if dtype == BF16 else 2.0 ** -22)
        inside("step", got, o, err + torch.finfo(dtype).eps / 2 * o.abs())
        near(lse, want_lse, F32, "lse", extra=2.0 ** -18)
        now = [n + 1 for n in now]
    assert ctx.device_status() == 0 and math.isfinite(float(got.float().sum()))
