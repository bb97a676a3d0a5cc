"""A tensor of another device is refused before its address reaches a kernel, also by a call that otherwise looks like one that
has been made (no GPU: tensors that say where they are)."""
import pytest
import torch

from tests.test_stream_memory_cpu import Memory, m, world  # noqa: F401


class There(Memory):
    device = torch.device("cuda", 1)

    def get_device(self):
        return 1


def there(t):
    return There(t.t, t.owner)


def arguments():
    x, st = m(2, 5, 8), m(2, 8)
    q, k = m(2, 5, 4, 64), m(2, 5, 2, 64)
    q1, k1, k_cache, v_cache = m(2, 4, 64), m(2, 2, 64), m(2, 5, 2, 64), m(2, 5, 2, 64)
    pos, lse, table = m(2, dtype=torch.int32), m(2, 4, 5), m(9, 16, 2)
    return dict(
        lasad_scan_forward=dict(x=x, gate=x, h_in=st, y=x, h_out=st),
        lasad_scan_backward=dict(x=x, gate=x, saved=m(2, 1, 8), dy=x, dh_out=st, dx=x, dgate=x, dh_in=st),
        lasad_scan_step=dict(x=m(2, 8), gate=m(2, 8), h_in=st, pos=pos, h_out=m(2, 8)),
        lasad_qk_norm_rope=dict(q=q, k=k, table=table, q_weight=m(64), k_weight=m(64), pos=pos, grid_w=3),
        lasad_qk_norm_rope_backward=dict(q=q, k=k, table=table, dq_out=q, dk_out=k, pos=pos, dq=q, dk=k, grid_w=3),
        lasad_window_attention=dict(q=q, k=k, v=k, lengths=pos, o=q, lse=lse, window=4),
        lasad_window_attention_backward=dict(q=q, k=k, v=k, o=q, lse=lse, do=q, lengths=pos, dq=q, dk=k, dv=k, window=4,
                                             workspace=m(64)),
        lasad_window_attention_step=dict(q=q1, k=k1, v=k1, k_cache=k_cache, v_cache=v_cache, pos=pos, window=4, sinks=1, o=q1),
        lasad_window_cache_store=dict(k=k, v=k, k_cache=k_cache, v_cache=v_cache, lengths=pos, window=4, sinks=1),
    )


@pytest.mark.parametrize("call,name", [(c, n) for c, kw in arguments().items() for n, t in kw.items() if isinstance(t, Memory)])
@pytest.mark.parametrize("made_before", [False, True])
def test_a_tensor_of_another_device_is_refused(world, call, name, made_before):      # noqa: F811
    ctx, _ = world
    kw = arguments()[call]
    if made_before:
        getattr(ctx, call)(**kw)
    with pytest.raises(ValueError):
        getattr(ctx, call)(**{**kw, name: there(kw[name])})
