"""An error that another call of the thread left behind (here: a device that is not there was asked for) is not the
library's: calls go through, and what was left is still there for whoever looks for it."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def leave_error(gpu):
    """Leaves an error with the HIP runtime that torch loaded; the status that a reader of it gets."""
    import torch
    torch.zeros(1, device="cuda")
    path = next(l.split()[-1] for l in open("/proc/self/maps") if "libamdhip64" in l)
    hip = C.CDLL(path)

    def leave():
        torch.cuda.synchronize()
        status = hip.hipSetDevice(9999)
        assert status != 0
        return status
    leave.last, leave.clear = hip.hipPeekAtLastError, hip.hipGetLastError
    yield leave
    hip.hipGetLastError()


def test_training_operators(leave_error):
    import torch
    import paper_2609_31224_amd as a2t
    n = 40
    q, k, v = torch.randn((n, 4, 64), device="cuda"), torch.randn((n, 2, 64), device="cuda"), torch.randn((n, 2, 64), device="cuda")
    pos, until = torch.arange(n, dtype=torch.int32, device="cuda"), torch.full((n,), 30, dtype=torch.int32, device="cuda")
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty((4, n), device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    logits, target, losses, logp = torch.randn((n, 64), device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda"), torch.empty(n, device="cuda")
    grad = torch.empty_like(logits)
    rope, prompt = a2t.a2t_rope_create(64, a2t.A2T_F32), a2t.a2t_prompt_create(n, 4, 2, 64, a2t.A2T_F32, flags=a2t.A2T_PROMPT_UNTIL)
    prefer = a2t.a2t_prefer_create(n, 64, a2t.A2T_F32)
    calls = [lambda: a2t.a2t_rope_apply(rope, pos, q, k, q, k), lambda: a2t.a2t_prompt_attn(prompt, [30, 10], q, k, v, o, lse, until),
             lambda: a2t.a2t_prompt_attn_grad(prompt, [30, 10], q, k, v, o, lse, q, dq, dk, dv, until), lambda: a2t.a2t_prefer_logp(prefer, logits, target, logp),
             lambda: a2t.a2t_prefer_loss(prefer, [15, 25], logits, target, losses, ref_logp=logp, grad=grad)]
    try:
        for call in calls:
            for _ in range(2):
                left = leave_error()
                call()
                assert leave_error.last() == left
                leave_error.clear()
        torch.cuda.synchronize()
        assert torch.isfinite(dq).all() and torch.isfinite(losses).all()
    finally:
        a2t.a2t_rope_destroy(rope)
        a2t.a2t_prompt_destroy(prompt)
        a2t.a2t_prefer_destroy(prefer)


@pytest.mark.parametrize("dtype", ["A2T_F32", "A2T_BF16", "A2T_MX4"])
def test_caches(leave_error, dtype):
    """A stream's steps: rows, chunk and single-row attention, eviction and the rows read back."""
    import torch
    import paper_2609_31224_amd as a2t
    dt = torch.float32 if dtype == "A2T_F32" else torch.bfloat16
    c = a2t.a2t_cache_create(1, 1, 4, 2, 64, getattr(a2t, dtype), 400, 100, 40)
    k, v, q, o = (torch.randn((1, 40, h, 64), device="cuda").to(dt) for h in (2, 2, 4, 4))
    seg = [a2t.SEG_ACOUSTIC] * 30 + [a2t.SEG_DELIM] + [a2t.SEG_TEXT] * 8 + [a2t.SEG_DELIM]
    steps = 8
    try:
        for unit in range(steps):
            pos = list(range(40 * unit, 40 * unit + 40))
            for call in (lambda: a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, [0], [40], k, v, seg, pos, [unit]), lambda: a2t.a2t_chunk_attn(c, 0, [0], [40], q, o),
                         lambda: a2t.a2t_decode_attn(c, 0, [0], q[0, :1], o[0, :1]), lambda: a2t.a2t_evict(c, [0], 200, 2), lambda: a2t.a2t_sync(c)):
                left = leave_error()
                call()
                assert leave_error.last() in (left, 0)       # waiting for the GPU may clear it
                leave_error.clear()
        assert a2t.a2t_resident(c, 0)[0] < 40 * steps and torch.isfinite(o.float()).all()
    finally:
        a2t.a2t_cache_destroy(c)


def test_adaptation_objective(leave_error):
    import torch
    import paper_2609_31224_amd as a2t
    from synth.distill import make_distill_batch
    b = make_distill_batch(seed=11, n_utt=2, units=3, vocab=200, added=2, dtype="f32")
    s, t = torch.randn((b.n, 208), device="cuda"), torch.randn((b.n, 200), device="cuda")
    losses, grad = torch.zeros(5, device="cuda"), torch.zeros_like(s)
    d = a2t.a2t_distill_create(b.n, 200, 2, a2t.A2T_F32)
    try:
        for _ in range(2):
            left = leave_error()
            a2t.a2t_distill_loss(d, s, t, b.kind, b.target, b.dec_group, b.turn_group, 1.0, losses, grad)
            assert leave_error.last() in (left, 0)
            leave_error.clear()
        torch.cuda.synchronize()
        assert torch.isfinite(losses).all()
    finally:
        a2t.a2t_distill_destroy(d)
