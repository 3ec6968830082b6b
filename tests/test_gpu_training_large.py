"""Variants of the training operators that large inputs select: rotary encoding with four and eight rows a workgroup and
outputs stored past the caches; preference losses whose first rows are streamed and whose last stay in the caches, wide
rows, rows far apart, strides with whole chunks of padding and different ones for policy and reference."""
import numpy as np
import pytest

from oracle.rope_forms import frequencies
from tests.test_gpu_prefer import U, _handle
from tests.test_gpu_rope import _check, _handle as _rope, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n,hq,hkv,d,part,dtype", [(4099, 3, 1, 64, 64, "bf16"), (8195, 2, 2, 128, 96, "f32"), (16385, 8, 2, 128, 128, "bf16"), (4099, 16, 4, 128, 64, "f32"),
                                                   (70001, 2, 2, 64, 48, "bf16")])
def test_rope(gpu, n, hq, hkv, d, part, dtype, pairs):
    """All rows against the same rows in calls of 700, which other tests hold against the oracle, bit for bit;
    some against the oracle itself; in place as out of place, and the gradient."""
    import torch
    import paper_2609_31224_amd as a2t
    rng = np.random.default_rng(n)
    freq, m = frequencies(part, 1e6, "yarn", 32.0, 4096)
    r = _rope(d, dtype, part, pairs, "yarn")
    try:
        both = _rows(rng, n, hq + hkv + 1, d, dtype)
        q, k = both[:, :hq], both[:, hq:hq + hkv]
        pos = rng.integers(0, 100000, n).astype(np.int32)
        p = torch.from_numpy(pos).to("cuda")
        some = np.unique(np.concatenate([np.arange(9), rng.integers(0, n, 60), n - 1 - np.arange(9)]))
        at = torch.from_numpy(some).to("cuda")
        for back in (False, True):
            outs = [torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda") for x in (q, k)]
            want = [torch.full_like(x, 7.0) for x in outs]
            a2t.a2t_rope_apply(r, p, q, k, *outs, grad=back)
            for lo in range(0, n, 700):
                w = slice(lo, min(lo + 700, n))
                a2t.a2t_rope_apply(r, p[w], q[w], k[w], want[0][w], want[1][w], grad=back)
            torch.cuda.synchronize()
            for x, y, z in zip(outs, want, (q, k)):
                assert torch.equal(x, y)
                _check(x[at], z[at], pos[some], freq, m, pairs, back, dtype)
        rest = both[:, hq + hkv:].clone()
        a2t.a2t_rope_apply(r, p, q, k, q, k, grad=True)
        torch.cuda.synchronize()
        assert torch.equal(q, outs[0]) and torch.equal(k, outs[1]) and torch.equal(both[:, hq + hkv:], rest)
    finally:
        a2t.a2t_rope_destroy(r)


def _prefer(rows, vocab, policy_stride, reference_stride, dtype, given, smoothing, in_place=False):
    """One call with a gradient against torch in 64 bits on the GPU, all rows: a row's log probability within
    2^-20 + 2^-23 of its largest logit, and what follows from it (test_gpu_prefer.py)."""
    import torch
    import paper_2609_31224_amd as a2t
    n, beta = sum(rows), 0.05
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator("cuda").manual_seed(vocab)

    def logits(stride):
        x = torch.empty((n, stride), dtype=dt, device="cuda")
        for lo in range(0, n, 256):
            x[lo:lo + 256, :vocab] = 2.0 * torch.randn((min(256, n - lo), vocab), device="cuda", generator=gen)
        x[:, vocab:vocab + 64] = float("nan")
        x[:, -64:][:, max(0, 64 - (stride - vocab)):] = float("nan")
        return x
    pol, ref = logits(policy_stride), None if given else logits(reference_stride)
    target = torch.randint(vocab, (n,), device="cuda", generator=gen, dtype=torch.int32)
    target[::11] = -100
    used = target >= 0
    top = 0.0

    def token_logp(x):
        nonlocal top
        out = []
        for lo in range(0, n, 128):
            y = x[lo:lo + 128, :vocab].double()
            top = max(top, float(y.abs().max()))
            out.append(torch.log_softmax(y, -1).gather(1, target[lo:lo + 128].clamp(min=0).long()[:, None])[:, 0])
        return torch.where(used, torch.cat(out), 0.0)
    p64 = token_logp(pol)
    r64 = (p64 - 0.01 * torch.rand(n, device="cuda", generator=gen)).float().double() if given else token_logp(ref)
    answer = torch.from_numpy(np.repeat(np.arange(len(rows)), rows)).to("cuda")
    ratios64 = torch.zeros(len(rows), dtype=torch.float64, device="cuda").index_add_(0, answer, torch.where(used, p64 - r64, 0.0))
    h64 = beta * (ratios64[0::2] - ratios64[1::2])
    sig = torch.nn.functional.logsigmoid
    loss64 = -((1 - smoothing) * sig(h64) + smoothing * sig(-h64)).mean()
    c = beta * ((1 - smoothing) * torch.sigmoid(-h64) - smoothing * torch.sigmoid(h64)) / len(h64)
    slope = torch.where(used, torch.stack([c, -c], -1).flatten()[answer], 0.0)
    losses, ratios = torch.full((3,), 7.0, device="cuda"), torch.full((len(rows),), 7.0, device="cuda")
    keep = pol.clone() if in_place else pol
    grad = pol if in_place else torch.full((n, policy_stride), 7.0, dtype=dt, device="cuda")
    h = _handle(n, vocab, dtype)
    try:
        a2t.a2t_prefer_loss(h, rows, pol, target, losses, ref, r64.float() if given else None, beta, smoothing, ratios, grad)
        torch.cuda.synchronize()
    finally:
        a2t.a2t_prefer_destroy(h)
    per_row = 2.0 ** -20 + 2.0 ** -23 * top
    off = per_row * 2 * torch.tensor(rows, device="cuda") + 2.0 ** -23 * ratios64.abs()
    assert ((ratios.double() - ratios64).abs() <= off).all()
    h_off = float(beta * (off[0::2] + off[1::2]).max() + 2.0 ** -23 * (h64.mean().abs() + loss64.abs()))
    assert abs(float(losses[0] - loss64)) <= h_off and abs(float(losses[1] - h64.mean())) <= h_off
    rel = U[dtype] + 2.0 ** -19 + 4 * h_off + per_row
    for lo in range(0, n, 128):
        w = slice(lo, min(lo + 128, n))
        p = torch.softmax(keep[w, :vocab].double(), -1)
        p[torch.arange(len(p), device="cuda"), target[w].clamp(min=0).long()] -= 1.0
        want = slope[w][:, None] * p
        tol = rel * want.abs() + (2.0 ** -23 + 4 * h_off) * slope[w].abs()[:, None] + 2.0 ** -133
        assert ((grad[w, :vocab].double() - want).abs() <= tol).all(), lo
        assert not grad[w, vocab:].any(), lo


@pytest.mark.parametrize("case", [
    # rows, vocabulary, strides, type, reference as log probabilities, smoothing, in place
    ([450, 431, 2, 460, 520, 477, 301, 130], 32005, 32008, 32064, "bf16", False, 0.0, False),       # 177 MB: the first 150 rows streamed
    ([450, 431, 2, 460, 520, 477, 301, 130], 32005, 32064, 32008, "bf16", True, 0.1, True),
    ([50] * 12, 151938, 151944, 151968, "bf16", False, 0.1, False),                                 # 182 MB, wide rows
    ([160, 170, 300, 90, 240, 410], 32005, 32032, 32008, "f32", False, 0.0, False),                 # 176 MB
    ([120, 30, 20, 70], 70001, 70008 + 4096, 70008 + 8, "f32", True, 0.0, True)])
def test_prefer_streamed_and_strided(gpu, case):
    _prefer(*case)


@pytest.mark.parametrize("rows,vocab,ps,rs,dtype", [([3, 5], 61, 64 + 8 * 300, 64, "bf16"), ([3, 5], 61, 64, 64 + 8 * 5, "f32"), ([100, 120], 203, 208 + 8 * 40, 208 + 16, "bf16"),
                                                    ([7, 9], 40001, 40008 + 2048 * 8, 40016, "f32")])
def test_prefer_padding(gpu, rows, vocab, ps, rs, dtype):
    """Strides with whole chunks of padding, which holds NaN in the logits and is zero in the gradient."""
    for given in (False, True):
        for in_place in (False, True):
            _prefer(rows, vocab, ps, rs, dtype, given, 0.1, in_place)


def test_prefer_rows_far_apart(gpu):
    """Rows 2^30 elements apart, whose offsets pass 32 bits, in bytes and in elements: the loss, the ratios and the
    gradient of the same rows side by side, bit for bit, and zeros in between."""
    import torch
    import paper_2609_31224_amd as a2t
    n, vocab, apart = 5, 997, 2 ** 30
    dense = torch.randn((n, 1000), device="cuda").to(torch.bfloat16)
    wide = torch.empty((n, apart), dtype=torch.bfloat16, device="cuda")        # 10 GB, the gradient as much
    wide[:, :1000] = dense
    grad_wide = torch.ones_like(wide)
    target, lp = torch.arange(n, dtype=torch.int32, device="cuda"), torch.full((n,), -6.0, device="cuda")
    h = _handle(n, vocab, "bf16")
    try:
        got = []
        for x, g in ((dense, torch.empty_like(dense)), (wide, grad_wide)):
            losses, ratios = torch.empty(3, device="cuda"), torch.empty(2, device="cuda")
            a2t.a2t_prefer_loss(h, [2, 3], x, target, losses, x, ratios=ratios, grad=g)
            a2t.a2t_prefer_loss(h, [2, 3], x, target, losses, ref_logp=lp, ratios=ratios, grad=g)
            torch.cuda.synchronize()
            got.append([losses, ratios, g[:, :1000].clone()])
        assert all(torch.equal(x, y) and torch.isfinite(x).all() for x, y in zip(*got))
        assert all(not row[1000:].view(torch.int16).any() for row in grad_wide)
    finally:
        a2t.a2t_prefer_destroy(h)
