"""Refusals of the operators for training on whole sessions that need no GPU: sizes and values are checked
before a device is looked for, calls without a handle are refused, and without a device a handle is not made."""
import ctypes as C

import pytest

import paper_2609_31224_amd as a2t

INVALID, NODEV = a2t.A2T_ERR_INVALID, a2t.A2T_ERR_NODEV


def _status(call, *args, **kw):
    with pytest.raises(a2t.A2TError) as e:
        call(*args, **kw)
    return e.value.status


def _no_gpu():
    import torch
    return not torch.cuda.is_available()


@pytest.mark.parametrize("kw", [dict(head_dim=32), dict(dtype=a2t.A2T_MX4), dict(rotary_dim=8), dict(rotary_dim=72), dict(rotary_dim=-16), dict(layout=-1),
                                dict(scaling=-1), dict(scaling=9), dict(theta=-1.0), dict(theta=float("nan")), dict(scaling=2, factor=float("inf")),
                                dict(scaling=3, factor=2.0, trained_rows=0), dict(scaling=3, factor=2.0, trained_rows=10, turns_slow=0.0)])
def test_rope_create(kw):
    args = dict(head_dim=64, dtype=a2t.A2T_BF16)
    args.update(kw)
    assert _status(a2t.a2t_rope_create, **args) == INVALID


@pytest.mark.parametrize("args,kw", [((0, 4, 2, 64, 1), {}), ((8, 4, 0, 64, 1), {}), ((8, 6, 4, 64, 1), {}), ((8, 4, 2, 80, 1), {}), ((8, 4, 2, 64, 3), {}),
                                     ((8, 4, 2, 64, 1), dict(flags=4)), ((8, 4, 2, 64, 1), dict(attn_scale=1e-9)), ((8, 4, 2, 64, 1), dict(attn_scale=float("inf"))),
                                     ((2**26 + 1, 1, 1, 64, 1), {}), ((2**26, 16, 1, 64, 1), {}), ((8, 4097, 4097, 64, 1), {}), ((2**31 - 1, 2**31 - 1, 1, 64, 1), {}), ((8, 258, 2, 64, 1), {})])
def test_prompt_create(args, kw):
    assert _status(a2t.a2t_prompt_create, *args, **kw) == INVALID


@pytest.mark.parametrize("args", [(0, 8, 1), (-1, 8, 1), (8, 0, 1), (8, 8, 2), (2**22 + 1, 8, 0), (8, 2**30 + 1, 0)])
def test_prefer_create(args):
    assert _status(a2t.a2t_prefer_create, *args) == INVALID


def test_without_a_device_or_a_handle():
    lib = a2t.raw_lib()
    if _no_gpu():
        assert _status(a2t.a2t_rope_create, 64, a2t.A2T_BF16) == NODEV
        assert _status(a2t.a2t_prompt_create, 8, 4, 2, 64, a2t.A2T_BF16) == NODEV
        assert _status(a2t.a2t_prefer_create, 8, 100, a2t.A2T_F32) == NODEV
    one = (C.c_int32 * 2)(1, 1)
    assert lib.a2t_rope_create(None, None, None) == INVALID
    out = C.c_void_p(1)
    assert lib.a2t_rope_create(None, None, C.byref(out)) == INVALID and not out.value
    assert lib.a2t_rope_apply(None, 1, None, 1, None, 64, None, 64, 0, None, 0, None, 0, 0) == INVALID
    assert lib.a2t_prompt_create(8, 4, 2, 64, 1, 0.0, 0, 0, None, None) == INVALID
    assert lib.a2t_prompt_attn(None, 1, one, None, 0, None, 0, None, 0, None, None, None) == INVALID
    assert lib.a2t_prompt_attn_grad(None, 1, one, None, 0, None, 0, None, 0, None, None, None, None, None, None, None) == INVALID
    assert lib.a2t_prefer_create(8, 8, 0, 0, None, None) == INVALID
    assert lib.a2t_prefer_logp(None, 1, None, 8, None, None) == INVALID
    assert lib.a2t_prefer_loss(None, 1, one, None, 8, None, 8, None, None, 0.1, 0.0, None, None, None) == INVALID
    for name in ("rope", "prompt", "prefer"):
        assert getattr(lib, f"a2t_{name}_destroy")(None) == INVALID
        assert getattr(lib, f"a2t_{name}_set_stream")(None, None) == INVALID


def test_tensors_in_host_memory():
    import torch
    x, i = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(8)
    rope, prompt, prefer = a2t.Rope(C.c_void_p(), 64, a2t.A2T_F32), a2t.Prompt(C.c_void_p(), 4, 2, 2, 64, a2t.A2T_F32), a2t.Prefer(C.c_void_p(), 4, 64, a2t.A2T_F32)
    for call in (lambda: a2t.a2t_rope_apply(rope, i, x, None, x), lambda: a2t.a2t_prompt_attn(prompt, [4], x, x, x, x, f),
                 lambda: a2t.a2t_prompt_attn_grad(prompt, [4], x, x, x, x, f, x, x, x, x),
                 lambda: a2t.a2t_prefer_logp(prefer, x[:, 0], i, f[:4]), lambda: a2t.a2t_prefer_loss(prefer, [2, 2], x[:, 0], i, f[:3], ref_logp=f[:4])):
        with pytest.raises(ValueError, match="GPU"):
            call()
