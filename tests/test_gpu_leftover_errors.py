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
