"""The oracles of the operators for training on whole sessions, pinned: attention over packed
sequences against torch's float64 autograd and against differences; rotary forms against their
definitions, the transposed map and the cache oracle's encoding; the preference loss against torch."""
import numpy as np
import pytest
import torch

from oracle import rope
from oracle.prefer import prefer_loss, token_logp
from oracle.prompt import prompt_attention, visible
from oracle.rope_forms import frequencies, rotate


def _attn_inputs(seed, n, hq, hkv, d):
    r = np.random.default_rng(seed)
    return [r.standard_normal((n, h, d)) for h in (hq, hkv, hkv, hq)]


@pytest.mark.parametrize("lengths,until", [([5], None), ([3, 0, 4], None), ([6], "some"), ([4, 5], "none")])
def test_attention_against_autograd_and_differences(lengths, until):
    n, hq, hkv, d = sum(lengths), 4, 2, 6
    q, k, v, do = _attn_inputs(1, n, hq, hkv, d)
    r = np.random.default_rng(2)
    ut = None if until is None else r.integers(-1, max(lengths) + 2, n) if until == "some" else np.zeros(n, int)
    got = prompt_attention(lengths, q, k, v, ut, do, scale=0.3)

    def forward(q, k, v):
        out, at = [], 0
        for m in lengths:
            see = torch.from_numpy(visible(m, None if ut is None else ut[at:at + m]))
            heads = []
            for h in range(hq):
                s = 0.3 * q[at:at + m, h] @ k[at:at + m, h // 2].T
                e = torch.where(see, torch.exp(torch.where(see, s, 0.0)), 0.0)
                z = e.sum(1, keepdim=True)
                heads.append(e / torch.where(z > 0, z, 1.0) @ v[at:at + m, h // 2])
            out.append(torch.stack(heads, 1))
            at += m
        return torch.cat(out)

    t = [torch.from_numpy(x).requires_grad_() for x in (q, k, v)]
    o = forward(*t)
    assert np.allclose(o.detach().numpy(), got.o, atol=1e-12)
    want = torch.autograd.grad(o, t, torch.from_numpy(do), allow_unused=True)
    for c, w in zip(("dq", "dk", "dv"), want):
        assert np.allclose(w.numpy(), got.grads[c], atol=1e-11), c
    # differences of sum(dO O) along one direction of every input
    eps = 1e-6
    dirs = [r.standard_normal(x.shape) for x in (q, k, v)]
    up, down = (prompt_attention(lengths, *(x + s * eps * y for x, y in zip((q, k, v), dirs)), ut, scale=0.3).o for s in (1, -1))
    slope = (do * (up - down)).sum() / (2 * eps)
    assert abs(slope - sum((got.grads[c] * y).sum() for c, y in zip(("dq", "dk", "dv"), dirs))) < 1e-6


def test_attention_rows():
    q, k, v, do = _attn_inputs(3, 5, 1, 1, 4)
    got = prompt_attention([5], q, k, v, np.array([1, 1, 9, 9, 3]), do)
    assert np.array_equal(got.o[0, 0], v[0, 0])                       # a row that sees itself alone
    assert not got.o[1].any() and got.lse[0, 1] == -np.inf           # the first row is gone, its own never there
    assert np.array_equal(got.o[2, 0], v[2, 0])
    assert not got.grads["dk"][[1, 4]].any() and not got.grads["dv"][[1, 4]].any() and not got.grads["dq"][1].any()
    for b in got.bounds.values():
        assert (b >= 0).all() and np.isfinite(b).all()


def test_rotary_forms():
    f, m = frequencies(64, 1e4)
    assert m == 1 and f[0] == 1 and abs(f[-1] - 1e4 ** (-62 / 64)) < 1e-15
    x = np.random.default_rng(4).standard_normal((3, 2, 64))
    pos = np.array([0, 5, 70000])
    f6, _ = frequencies(64, 1e6)
    ref = np.stack([rope.rotate(x[:, h], pos, 1e6) for h in range(2)], 1)
    assert np.allclose(rotate(x, pos, f6), ref, atol=1e-9)           # the caches' encoding
    assert np.allclose(frequencies(64, 1e4, "linear", 4.0)[0], f / 4)
    ntk = frequencies(64, 1e4, "ntk", 4.0)[0]
    assert ntk[0] == 1 and abs(ntk[-1] - f[-1] / 4) < 1e-12          # the slowest pair is interpolated, the fastest kept
    y, m = frequencies(64, 1e4, "yarn", 4.0, 4096)
    assert abs(m - (0.1 * np.log(4) + 1)) < 1e-15
    turns = 4096 * f / (2 * np.pi)
    assert np.array_equal(y[turns > 40], f[turns > 40]) and np.allclose(y[turns < 0.5], f[turns < 0.5] / 4)
    assert (np.diff(y) < 0).all()
    for pairs in (False, True):      # the transposed map: <R x, y> = <x, R' y>; part of the head
        g = np.random.default_rng(5).standard_normal(x.shape)
        fr = frequencies(32, 1e4)[0]
        a = (rotate(x, pos, fr, 1.2, pairs) * g).sum()
        assert abs(a - (x * rotate(g, pos, fr, 1.2, pairs, back=True)).sum()) < 1e-10
        assert np.array_equal(rotate(x, pos, fr, 1.2, pairs)[..., 32:], x[..., 32:])


@pytest.mark.parametrize("smoothing,given", [(0.0, False), (0.2, True)])
def test_preference_loss(smoothing, given):
    rows, vocab, r = [3, 2, 0, 4], 11, np.random.default_rng(6)
    pol, ref = 2 * r.standard_normal((9, vocab)), 2 * r.standard_normal((9, vocab))
    target = r.integers(0, vocab, 9)
    target[[1, 5]] = -100, vocab
    kw = dict(ref_logp=token_logp(ref, target)) if given else dict(reference=ref)
    got = prefer_loss(rows, pol, target, beta=0.7, smoothing=smoothing, **kw)
    t = torch.from_numpy(pol).requires_grad_()
    used = [i for i in range(9) if i not in (1, 5)]
    lp = torch.log_softmax(t, -1)
    lr = torch.log_softmax(torch.from_numpy(ref), -1)
    d = torch.zeros(9, dtype=torch.float64)
    for i in used:
        d[i] = lp[i, target[i]] - lr[i, target[i]]
    a = [d[0:3].sum(), d[3:5].sum(), d[5:5].sum(), d[5:9].sum()]
    h = torch.stack([0.7 * (a[0] - a[1]), 0.7 * (a[2] - a[3])])
    ls = torch.nn.functional.logsigmoid
    loss = -((1 - smoothing) * ls(h) + smoothing * ls(-h)).mean()
    loss.backward()
    assert abs(loss.item() - got.loss) < 1e-12 and abs(h.mean().item() - got.margin) < 1e-12
    assert np.allclose(t.grad.numpy(), got.grad, atol=1e-13) and got.won == (h > 0).double().mean().item()
    assert not got.grad[[1, 5]].any()
    eps, y = 1e-6, r.standard_normal(pol.shape)
    up, down = (prefer_loss(rows, pol + s * eps * y, target, beta=0.7, smoothing=smoothing, **kw).loss for s in (1, -1))
    assert abs((up - down) / (2 * eps) - (got.grad * y).sum()) < 1e-8
