"""Outputs of the preference loss over its inputs and over each other: refused where other workgroups read what
would be written; the gradient over the policy's logits, or over the reference's, has the same bits as elsewhere."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu


def test_refusals_and_in_place(gpu):
    import torch
    import paper_2609_31224_amd as a2t
    lib, n, vocab, S = a2t.raw_lib(), 10, 60, 64
    h = a2t.a2t_prefer_create(n, vocab, a2t.A2T_F32)
    # operands far from each other in one room: every call below stays within it
    room = torch.zeros((16 * n, S), device="cuda")
    at = lambda i: room[i * n:(i + 1) * n]  # noqa: E731
    pol, ref, grad = at(2), at(4), at(6)
    pol.copy_(torch.randn(pol.shape, device="cuda"))
    ref.copy_(torch.randn(pol.shape, device="cuda"))
    flat = lambda i, m: at(i).view(-1)[:m]  # noqa: E731
    target, lp, losses, ratios, logp = flat(8, n).view(torch.int32), flat(9, n), flat(10, 3), flat(11, 4), flat(12, n)
    target.copy_(torch.arange(n))
    lp.fill_(-4.0)
    keep = room.clone()
    p = {k: v.data_ptr() for k, v in dict(pol=pol, ref=ref, grad=grad, target=target, lp=lp, losses=losses, ratios=ratios, logp=logp).items()}
    rows, row = (C.c_int32 * 4)(3, 2, 1, 4), S * 4

    def loss(given=False, **kw):
        a = {**p, **kw}
        ref, lp = (None, a["lp"]) if given else (a["ref"], None)
        return lib.a2t_prefer_loss(h.ptr, 2, rows, a["pol"], S, ref, S, lp, a["target"], 0.1, 0.0, a["losses"], a["ratios"], a["grad"])

    def score(**kw):
        a = {**p, **kw}
        return lib.a2t_prefer_logp(h.ptr, n, a["pol"], S, a["target"], a["logp"])
    try:
        for given, bad in ((False, dict(grad=p["pol"] + row)), (False, dict(grad=p["pol"] - row)), (False, dict(grad=p["pol"] + 16)), (False, dict(grad=p["pol"] + 9 * row)),
                           (False, dict(grad=p["target"])), (False, dict(grad=p["target"] - 9 * row)), (True, dict(grad=p["lp"])), (False, dict(losses=p["pol"] + 8)),
                           (False, dict(losses=p["pol"] + 9 * row + 236)), (False, dict(losses=p["target"] + 32)), (True, dict(losses=p["lp"] + 36)), (False, dict(losses=p["ref"])),
                           (False, dict(ratios=p["pol"])), (False, dict(ratios=p["target"])), (True, dict(ratios=p["lp"] - 12)), (False, dict(losses=p["ratios"] + 8)),
                           (False, dict(losses=p["ratios"] - 8)), (False, dict(losses=p["grad"] + 240)), (False, dict(ratios=p["grad"] + 9 * row + 240))):
            assert loss(given, **bad) == a2t.A2T_ERR_INVALID, bad
        for bad in (dict(logp=p["pol"] + 4), dict(logp=p["target"]), dict(logp=p["target"] - 36), dict(logp=p["pol"] + 9 * row + 236)):
            assert score(**bad) == a2t.A2T_ERR_INVALID, bad
        torch.cuda.synchronize()
        assert torch.equal(room, keep)
        assert loss() == a2t.A2T_OK and score() == a2t.A2T_OK
        torch.cuda.synchronize()
        want, values = grad.clone(), torch.cat([losses, ratios])
        for place in (ref, pol):
            room.copy_(keep)
            assert loss(grad=place.data_ptr()) == a2t.A2T_OK
            torch.cuda.synchronize()
            assert torch.equal(place, want) and torch.equal(torch.cat([losses, ratios]), values)
    finally:
        a2t.a2t_prefer_destroy(h)
