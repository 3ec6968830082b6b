"""Outputs of the attention over packed sequences that lie over its inputs: refused where another workgroup or a
later launch would read what was written, and the same bits as elsewhere where a row's reader is its writer."""
import ctypes as C

import pytest

from tests.test_gpu_prompt import _case, _like

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("until,sort,splits", [(None, 1, 0), (None, 1, 3), ("random", 1 << 20, 0), ("random", 1, 0), ("random", 1, 4), ("evicted", 1, 1)])
def test_in_place(gpu, monkeypatch, until, sort, splits, dtype, d):
    """o over q, then dq over o, dk over k and dv over v, for every form of the launches; 300 short sequences in two tables too."""
    import torch
    import paper_2609_31224_amd as a2t
    monkeypatch.setenv("A2T_PROMPT_SORT", str(sort))
    monkeypatch.setenv("A2T_PROMPT_SPLITS", str(splits))
    for lengths in ([290, 1, 66, 129], [3] * 300):
        n = sum(lengths)
        q, k, v, do, ut = _case(lengths, 4, 2, d, dtype, until, fused=False)
        ut = None if ut is None else torch.from_numpy(ut).to("cuda")
        h = a2t.a2t_prompt_create(n, 4, 2, d, a2t.A2T_F32 if dtype == "f32" else a2t.A2T_BF16, flags=0 if until is None else a2t.A2T_PROMPT_UNTIL)
        try:
            o, lse = torch.empty_like(q), torch.empty((4, n), device="cuda")
            grads = [torch.empty_like(x) for x in (q, k, v)]
            a2t.a2t_prompt_attn(h, lengths, q, k, v, o, lse, ut)
            a2t.a2t_prompt_attn_grad(h, lengths, q, k, v, o, lse, do, *grads, ut)
            over = q.clone()
            a2t.a2t_prompt_attn(h, lengths, over, k, v, over, None, ut)
            torch.cuda.synchronize()
            assert torch.equal(over, o)
            k2, v2 = k.clone(), v.clone()
            a2t.a2t_prompt_attn_grad(h, lengths, q, k2, v2, over, lse, do, over, k2, v2, ut)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip((over, k2, v2), grads))
            # parts of one projection, the keys' and values' in place
            both = torch.cat([q, k, v], 1)
            a2t.a2t_prompt_attn_grad(h, lengths, both[:, :4], both[:, 4:6], both[:, 6:], o, lse, do, _like(both[:, :4], 7.0), both[:, 4:6], both[:, 6:], ut)
            torch.cuda.synchronize()
            assert torch.equal(both[:, 4:6], grads[1]) and torch.equal(both[:, 6:], grads[2]) and torch.equal(both[:, :4], q)
        finally:
            a2t.a2t_prompt_destroy(h)


def test_refusals(gpu):
    """Every output over every other operand, whole and in part; nothing is written and the handle stays usable."""
    import torch
    import paper_2609_31224_amd as a2t
    lib, n = a2t.raw_lib(), 24
    h = a2t.a2t_prompt_create(n, 4, 2, 64, a2t.A2T_BF16, flags=a2t.A2T_PROMPT_UNTIL)
    # operands side by side, 2,048 elements a row, and others far from each other: every call below stays within the room
    room = torch.zeros((16 * n, 32, 64), dtype=torch.bfloat16, device="cuda")
    wide, S = room[4 * n:5 * n], 2048
    wide.copy_(torch.randn(wide.shape, device="cuda"))
    keep = wide.clone()
    part = lambda head: wide.data_ptr() + head * 64 * 2  # noqa: E731
    o, do, dq = (room[i * n:(i + 1) * n].view(-1)[:n * 256].view(n, 4, 64) for i in (8, 9, 10))
    lse, ut = (room[i * n:(i + 1) * n].view(-1).view(t)[:size].view(shape) for i, t, size, shape in ((11, torch.float32, 4 * n, (4, n)), (12, torch.int32, n, (n,))))
    ut.fill_(n)
    rows = (C.c_int32 * 2)(20, 4)
    base = dict(q=part(0), qs=S, k=part(4), v=part(6), until=ut.data_ptr(), o=o.data_ptr(), lse=lse.data_ptr())

    def attn(**kw):
        a = {**base, **kw}
        return lib.a2t_prompt_attn(h.ptr, 2, rows, a["q"], a["qs"], a["k"], S, a["v"], S, a["until"], a["o"], a["lse"])

    def grad(dq=part(8), dk=part(12), dv=part(14), **kw):
        a = {**base, **kw}
        return lib.a2t_prompt_attn_grad(h.ptr, 2, rows, a["q"], a["qs"], a["k"], S, a["v"], S, a["until"], a["o"], a["lse"], do.data_ptr(), dq, dk, dv)
    last = (n - 1) * S * 2
    try:
        bad = [dict(o=part(0)), dict(o=part(4)), dict(o=part(7)), dict(o=part(6) + last), dict(o=part(4) - (n - 1) * 512), dict(lse=part(0)), dict(lse=part(5) + last),
               dict(lse=o.data_ptr()), dict(lse=o.data_ptr() + n * 512 - 16), dict(lse=ut.data_ptr()), dict(o=ut.data_ptr() - 512), dict(o=lse.data_ptr() - n * 512 + 16),
               dict(q=o.data_ptr() + 16, qs=256), dict(q=o.data_ptr(), qs=264)]
        for kw in bad:
            assert attn(**kw) == a2t.A2T_ERR_INVALID, kw
        bad = [dict(dq=part(0)), dict(dq=part(1)), dict(dq=part(4)), dict(dq=part(3)), dict(dq=part(6)), dict(dk=part(0)), dict(dk=part(6)), dict(dk=part(5)), dict(dv=part(4)),
               dict(dv=part(5)), dict(dv=part(3)), dict(dk=part(8)), dict(dk=part(14)), dict(dv=part(11)), dict(dq=part(11)), dict(dk=o.data_ptr()), dict(dv=o.data_ptr() - last),
               dict(dk=do.data_ptr()), dict(dq=do.data_ptr()), dict(dq=o.data_ptr()), dict(dk=lse.data_ptr()), dict(dq=ut.data_ptr()),
               dict(qs=256, q=dq.data_ptr(), dq=do.data_ptr()), dict(qs=256, q=dq.data_ptr(), dq=dq.data_ptr()), dict(qs=256, q=dq.data_ptr(), dq=o.data_ptr() + 16)]
        for kw in bad:
            assert grad(**kw) == a2t.A2T_ERR_INVALID, kw
        torch.cuda.synchronize()
        assert torch.equal(wide, keep) and not any(x.any() for x in (o, do, dq, lse))
        # rows between each other's, and in place
        assert attn() == a2t.A2T_OK and grad() == a2t.A2T_OK
        assert grad(dk=part(4), dv=part(6)) == a2t.A2T_OK and grad(qs=256, q=dq.data_ptr(), dq=o.data_ptr()) == a2t.A2T_OK
        torch.cuda.synchronize()
        assert torch.equal(wide[:, 16:], keep[:, 16:]) and torch.equal(wide[:, :4], keep[:, :4])
        with pytest.raises(a2t.A2TError):
            a2t.a2t_prompt_attn_grad(h, [20, 4], dq, wide[:, 4:6], wide[:, 6:8], o, lse, do, dq, wide[:, 12:14], wide[:, 14:16])
        torch.cuda.synchronize()
    finally:
        a2t.a2t_prompt_destroy(h)


def test_operands_that_share_memory(gpu):
    """An output in place of one operand whose memory is another operand's too (keys that are the queries, a gradient of o that
    is o): refused; inputs may share memory as they like."""
    import torch
    import paper_2609_31224_amd as a2t
    n, lengths = 40, [30, 10]
    h = a2t.a2t_prompt_create(n, 2, 2, 64, a2t.A2T_F32)
    x, y, o, other = (torch.randn((n, 2, 64), device="cuda") for _ in range(4))
    lse, grads = torch.zeros((2, n), device="cuda"), [torch.zeros((n, 2, 64), device="cuda") for _ in range(3)]
    keep = [t.clone() for t in (x, y, o)]
    try:
        def refused(call, *args):
            with pytest.raises(a2t.A2TError) as e:
                call(h, lengths, *args)
            assert e.value.status == a2t.A2T_ERR_INVALID
        refused(a2t.a2t_prompt_attn, x, x, y, x)                # o over q, which is k
        refused(a2t.a2t_prompt_attn, x, y, x, x)                # and v
        for q, k, v, dq, dk, dv, d_o in ((x, x, y, grads[0], x, grads[2], other), (x, y, x, grads[0], grads[1], x, other), (x, y, y, grads[0], y, grads[2], other),
                                         (x, y, other, o, grads[1], grads[2], o), (o, x, y, o, grads[1], grads[2], other)):
            refused(a2t.a2t_prompt_attn_grad, q, k, v, o, lse, d_o, dq, dk, dv)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((x, y, o), keep)) and not any(g.any() for g in grads)
        got = []
        for q, k, v in ((x, x, x), (x.clone(), x.clone(), x.clone())):
            a2t.a2t_prompt_attn(h, lengths, q, k, v, o, lse)
            a2t.a2t_prompt_attn_grad(h, lengths, q, k, v, o, lse, o, *grads)
            torch.cuda.synchronize()
            got.append([t.clone() for t in (o, lse, *grads)])
        assert all(torch.equal(a, b) for a, b in zip(*got))
    finally:
        a2t.a2t_prompt_destroy(h)
