"""GPU parity of the preference loss (a2t_prefer_loss, a2t_prefer_logp) against the fp64 oracle.

A log probability is x - max - ln(sum): the sum's fp32 terms are off by 2^-20 of it at most (an
exponential 2 half steps and its argument's rounding, |x - max| 2^-24; partial sums of a thread's
share of the row), so a row's is off by 2^-20 + 2^-23 |logits|; an answer's ratio by that times its
rows, twice; the loss and h by beta times that.  A gradient element: half a step of its type, and
2^-19 of itself plus the slope's own error."""
import ctypes as C

import numpy as np
import pytest

from oracle.prefer import prefer_loss, token_logp

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _logits(rng, n, vocab, dtype, fill=np.nan):
    """[n][stride] on the GPU, the stride's padding filled; and what it holds, float64."""
    import torch
    stride = (vocab + 7) // 8 * 8
    x = np.full((n, stride), fill, np.float32)
    x[:, :vocab] = 2.0 * rng.standard_normal((n, vocab))
    t = torch.from_numpy(x).to("cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    return t, t[:, :vocab].cpu().double().numpy()


def _targets(rng, n, vocab):
    import torch
    t = rng.integers(0, vocab, n).astype(np.int32)
    return t, torch.from_numpy(t).to("cuda")


def _row_error(*logits):
    return 2.0 ** -20 + 2.0 ** -23 * max(np.abs(x).max() for x in logits)


def _check(got, ref, rows, beta, dtype, per_row):
    losses, ratios, grad, vocab = got
    off = per_row * 2 * np.asarray(rows) + 2.0 ** -23 * np.abs(ref.ratios)
    assert (np.abs(ratios - ref.ratios) <= off).all(), np.abs(ratios - ref.ratios).max()
    h_off = beta * (off[0::2] + off[1::2]).max() + 2.0 ** -23 * (abs(ref.margin) + abs(ref.loss))
    assert abs(losses[0] - ref.loss) <= h_off and abs(losses[1] - ref.margin) <= h_off
    assert abs(losses[2] - ref.won) <= 2.0 ** -24
    if grad is None:
        return
    assert not grad[:, vocab:].any()                # the stride's padding
    rel = U[dtype] + 2.0 ** -19 + 4 * h_off + per_row
    tol = rel * np.abs(ref.grad) + (2.0 ** -23 + 4 * h_off) * np.abs(ref.slope)[:, None] * (ref.grad != 0)
    tol += 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149     # results below the normal numbers
    assert (np.abs(grad[:, :vocab] - ref.grad) <= tol).all(), np.abs(grad[:, :vocab] - ref.grad).max()


def _run(h, rows, pol, target, ref=None, ref_logp=None, beta=0.1, smoothing=0.0, with_grad=True, in_place=False):
    import torch
    import paper_2609_31224_amd as a2t
    losses, ratios = torch.full((3,), 7.0, device="cuda"), torch.full((len(rows),), 7.0, device="cuda")
    g = None if not with_grad else pol if in_place else torch.full_like(pol, 7.0)
    a2t.a2t_prefer_loss(h, rows, pol, target, losses, ref, ref_logp, beta, smoothing, ratios, g)
    torch.cuda.synchronize()
    num = lambda x: None if x is None else x.cpu().double().numpy()  # noqa: E731
    return num(losses), num(ratios), num(g), h.vocab


def _handle(n, vocab, dtype, **kw):
    import paper_2609_31224_amd as a2t
    return a2t.a2t_prefer_create(n, vocab, a2t.A2T_F32 if dtype == "f32" else a2t.A2T_BF16, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,beta,smoothing", [
    ([1, 1], 1, 0.1, 0.0), ([2, 3], 7, 0.5, 0.1), ([0, 4, 5, 0], 8, 0.1, 0.0), ([3, 1, 70, 90], 997, 0.1, 0.2), ([17] * 6, 10007, 1.0, 0.0),
    ([5, 9], 40001, 0.1, 1.0), ([400, 700], 1031, 0.05, 0.0)])
def test_against_oracle(gpu, rows, vocab, beta, smoothing, dtype):
    import paper_2609_31224_amd as a2t
    import torch
    rng, n = np.random.default_rng(vocab), sum(rows)
    pol, p64 = _logits(rng, n, vocab, dtype)
    ref, r64 = _logits(rng, n, vocab, dtype)
    t, target = _targets(rng, n, vocab)
    if n > 8:
        t[::5] = -100                       # rows without a token of the answer
        t[3] = vocab
        target.copy_(torch.from_numpy(t))
    h = _handle(n + 3, vocab, dtype)
    try:
        want = prefer_loss(rows, p64, t, reference=r64, beta=beta, smoothing=smoothing)
        per_row = _row_error(p64, r64)
        _check(_run(h, rows, pol, target, ref, None, beta, smoothing), want, rows, beta, dtype, per_row)
        # the reference's log probabilities known, no gradient
        logp = torch.full((n,), 7.0, device="cuda")
        a2t.a2t_prefer_logp(h, ref, target, logp)
        torch.cuda.synchronize()
        assert (np.abs(logp.cpu().double().numpy() - token_logp(r64, t)) <= per_row + 2.0 ** -24 * 30).all()
        # rows without a token never read the reference
        logp[torch.from_numpy((t < 0) | (t >= vocab)).to("cuda")] = float("nan")
        _check(_run(h, rows, pol, target, None, logp, beta, smoothing, with_grad=False), want, rows, beta, dtype, per_row + 2.0 ** -24 * 30)
        # the gradient over the policy's own logits
        _check(_run(h, rows, pol, target, ref, None, beta, smoothing, in_place=True), want, rows, beta, dtype, per_row)
    finally:
        a2t.a2t_prefer_destroy(h)


def test_wide_vocabulary(gpu):
    """The extended vocabulary of 151,938 tokens, whose rows have a chunk of two logits at the end."""
    import paper_2609_31224_amd as a2t
    rows, vocab = [6, 5, 3, 4], 151938
    rng = np.random.default_rng(9)
    pol, p64 = _logits(rng, 18, vocab, "bf16")
    ref, r64 = _logits(rng, 18, vocab, "bf16")
    t, target = _targets(rng, 18, vocab)
    t[7] = vocab - 1
    target[7] = vocab - 1
    h = _handle(18, vocab, "bf16")
    try:
        _check(_run(h, rows, pol, target, ref), prefer_loss(rows, p64, t, reference=r64), rows, 0.1, "bf16", _row_error(p64, r64))
    finally:
        a2t.a2t_prefer_destroy(h)


def test_most_pairs_and_far_margins(gpu):
    """256 pairs of one row; margins of thousands, where the loss is the margin itself or zero."""
    import torch
    import paper_2609_31224_amd as a2t
    rng, rows, vocab = np.random.default_rng(10), [1] * 512, 64
    pol, p64 = _logits(rng, 512, vocab, "f32")
    t, target = _targets(rng, 512, vocab)
    lp = (token_logp(p64, t) + 3000.0 * np.sign(rng.standard_normal(512))).astype(np.float32)
    h = _handle(512, vocab, "f32")
    try:
        want = prefer_loss(rows, p64, t, ref_logp=lp, beta=2.0)
        assert want.loss > 100
        _check(_run(h, rows, pol, target, None, torch.from_numpy(lp).to("cuda"), 2.0), want, rows, 2.0, "f32", _row_error(p64) + 2.0 ** -24 * 3000)
    finally:
        a2t.a2t_prefer_destroy(h)


def test_masked_logits(gpu):
    """Tokens whose logits are -infinity have no weight and no gradient."""
    import paper_2609_31224_amd as a2t
    rng, rows, vocab = np.random.default_rng(11), [4, 4], 333
    pol, _ = _logits(rng, 8, vocab, "f32")
    t, target = _targets(rng, 8, 100)
    pol[:, 100:] = -np.inf
    ref = pol.clone()
    ref[:, :50] += 1
    h = _handle(8, vocab, "f32")
    try:
        p64, r64 = pol[:, :vocab].cpu().double().numpy(), ref[:, :vocab].cpu().double().numpy()
        want = prefer_loss(rows, p64, t, reference=r64)
        got = _run(h, rows, pol, target, ref)
        _check(got, want, rows, 0.1, "f32", _row_error(p64[:, :100], r64[:, :100]))
        assert not got[2][:, 100:].any()
    finally:
        a2t.a2t_prefer_destroy(h)


def test_gradient_against_differences(gpu):
    """The gradient against the library's own loss at logits moved both ways."""
    import torch
    import paper_2609_31224_amd as a2t
    rng, rows, vocab = np.random.default_rng(12), [3, 4], 50
    pol, _ = _logits(rng, 7, vocab, "f32", fill=0.0)
    ref, _ = _logits(rng, 7, vocab, "f32", fill=0.0)
    _, target = _targets(rng, 7, vocab)
    h = _handle(7, vocab, "f32")
    try:
        _, _, g, _ = _run(h, rows, pol, target, ref, beta=0.5)
        y = torch.randn(pol.shape, device="cuda")
        eps = 2.0 ** -6
        up, down = (_run(h, rows, pol + s * eps * y, target, ref, beta=0.5, with_grad=False)[0][0] for s in (1, -1))
        slope = (g * y.cpu().double().numpy()).sum()
        # third differences: eps^2 / 6 times a third derivative of order (7 beta)^3; losses are fp32
        assert abs((up - down) / (2 * eps) - slope) < eps ** 2 * 8 + 4 * 2.0 ** -24 / eps
    finally:
        a2t.a2t_prefer_destroy(h)


def test_same_results_and_rows_behind(gpu):
    """Bit by bit the same each time; rows past the last answer keep what they held."""
    import torch
    import paper_2609_31224_amd as a2t
    rng, rows, vocab = np.random.default_rng(13), [20, 31], 5003
    pol, _ = _logits(rng, 60, vocab, "bf16")
    ref, _ = _logits(rng, 60, vocab, "bf16")
    _, target = _targets(rng, 51, vocab)
    h = _handle(60, vocab, "bf16")
    try:
        a, b = (_run(h, rows, pol, target, ref) for _ in range(2))
        assert all(np.array_equal(x, y) for x, y in zip(a[:3], b[:3]))
        assert (a[2][51:] == 7).all()
    finally:
        a2t.a2t_prefer_destroy(h)


def test_captured_and_on_streams(gpu):
    import torch
    import paper_2609_31224_amd as a2t
    rng, rows, vocab = np.random.default_rng(14), [7, 9], 2003
    pol, _ = _logits(rng, 16, vocab, "bf16")
    ref, _ = _logits(rng, 16, vocab, "bf16")
    _, target = _targets(rng, 16, vocab)
    side = torch.cuda.Stream()
    h, other = _handle(16, vocab, "bf16", stream=side), _handle(16, vocab, "bf16")
    losses, ratios, grad = torch.zeros(3, device="cuda"), torch.zeros(4, device="cuda")[:2], torch.zeros_like(pol)
    try:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            a2t.a2t_prefer_loss(h, rows, pol, target, losses, ref, ratios=ratios, grad=grad)
        for turn in range(3):
            pol.copy_(torch.randn(pol.shape, device="cuda"))
            target.copy_(torch.randint(vocab, (16,), device="cuda", dtype=torch.int32))
            torch.cuda.synchronize()
            want = _run(other, rows, pol, target, ref)
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(losses.cpu().double().numpy(), want[0]) and np.array_equal(grad.cpu().double().numpy(), want[2]), turn
    finally:
        a2t.a2t_prefer_destroy(h)
        a2t.a2t_prefer_destroy(other)


def test_refusals(gpu):
    import torch
    import paper_2609_31224_amd as a2t
    lib = a2t.raw_lib()
    for args in ((0, 10, 1), (8, 0, 1), (8, 10, 2), (2**22 + 1, 10, 1), (8, 2**30 + 1, 1)):
        with pytest.raises(a2t.A2TError) as e:
            a2t.a2t_prefer_create(*args)
        assert e.value.status == a2t.A2T_ERR_INVALID
    h = _handle(8, 30, "f32")
    x, y = torch.zeros((8, 32), device="cuda"), torch.zeros((8, 32), device="cuda")
    t = torch.zeros(8, dtype=torch.int32, device="cuda")
    out = torch.zeros(16, device="cuda")
    o = out.data_ptr()

    def call(rows=(4, 4), pairs=None, pol=x.data_ptr(), ps=32, ref=y.data_ptr(), rs=32, lp=None, t=t.data_ptr(), beta=0.1, sm=0.0, losses=o, grad=None):
        r = np.array(rows, np.int32)
        return lib.a2t_prefer_loss(h.ptr, len(r) // 2 if pairs is None else pairs, r.ctypes.data_as(C.POINTER(C.c_int32)), pol, ps, ref, rs, lp, t, beta, sm, losses, None, grad)
    try:
        assert call() == a2t.A2T_OK
        for bad in (dict(rows=(4, 5)), dict(rows=(0, 0)), dict(rows=(9, -1)), dict(pairs=0), dict(pairs=-1), dict(pairs=257), dict(pol=None), dict(pol=x.data_ptr() + 4),
                    dict(ps=28), dict(ps=24), dict(rs=36), dict(ref=None), dict(lp=o), dict(t=None), dict(t=t.data_ptr() + 1), dict(beta=0.0), dict(beta=-1.0),
                    dict(beta=float("nan")), dict(sm=-0.1), dict(sm=1.1), dict(sm=float("nan")), dict(losses=None), dict(grad=x.data_ptr() + 4)):
            assert call(**bad) == a2t.A2T_ERR_INVALID, bad
        assert lib.a2t_prefer_logp(h.ptr, 9, x.data_ptr(), 32, t.data_ptr(), o) == a2t.A2T_ERR_INVALID
        assert lib.a2t_prefer_logp(h.ptr, 8, x.data_ptr(), 30, t.data_ptr(), o) == a2t.A2T_ERR_INVALID
        lo = out[:3]
        for bad in (lambda: a2t.a2t_prefer_loss(h, [4], x, t, lo, y), lambda: a2t.a2t_prefer_loss(h, [4, 4], x[:7], t, lo, y),
                    lambda: a2t.a2t_prefer_loss(h, [4, 4], x, t, lo, y.double()), lambda: a2t.a2t_prefer_loss(h, [4, 4], x, t[:7], lo, y),
                    lambda: a2t.a2t_prefer_loss(h, [4, 4], x, t, out[:2], y), lambda: a2t.a2t_prefer_loss(h, [4, 4], x[:, :29], t, lo, y),
                    lambda: a2t.a2t_prefer_loss(h, [4, 4], x, t, lo, y, grad=torch.zeros((8, 40), device="cuda"))):
            with pytest.raises(ValueError):
                bad()
        with pytest.raises(a2t.A2TError):
            a2t.a2t_prefer_loss(h, [4, 4], x, t, lo)          # neither a reference nor its log probabilities
        assert call() == a2t.A2T_OK
        torch.cuda.synchronize()
    finally:
        a2t.a2t_prefer_destroy(h)
