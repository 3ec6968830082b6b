"""The preference loss of long answers, whose ratios are formed in a launch of their own: against the
oracle within the limits of test_gpu_prefer.py, and in time that grows with the rows."""
import numpy as np
import pytest

from oracle.prefer import prefer_loss
from tests.test_gpu_prefer import _check, _handle, _logits, _row_error, _run, _targets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", [([95, 94], 61), ([0, 96], 61), ([96, 1, 0, 0, 3, 97], 61), ([4099, 3001], 203), ([1025] * 6, 17)])
def test_against_oracle(gpu, rows, vocab, dtype):
    """Longest answers on both sides of the rows from which the launch is made; empty and short ones beside them."""
    import torch
    import paper_2609_31224_amd as a2t
    rng, n = np.random.default_rng(sum(rows)), sum(rows)
    pol, p64 = _logits(rng, n, vocab, dtype)
    # a reference near the policy: margins stay where the slope is not flat
    ref = pol.clone()
    ref[:, ::3] += 2.0 ** -6
    r64 = ref[:, :vocab].cpu().double().numpy()
    t, target = _targets(rng, n, vocab)
    t[::7] = -1
    target.copy_(torch.from_numpy(t))
    h = _handle(n, vocab, dtype)
    try:
        want, per_row = prefer_loss(rows, p64, t, reference=r64, smoothing=0.1), _row_error(p64, r64)
        got = _run(h, rows, pol, target, ref, smoothing=0.1)
        _check(got, want, rows, 0.1, dtype, per_row)
        again, alone = _run(h, rows, pol, target, ref, smoothing=0.1), _run(h, rows, pol, target, ref, smoothing=0.1, with_grad=False)
        assert all(np.array_equal(x, y) for x, y in zip(got[:3], again[:3])) and all(np.array_equal(x, y) for x, y in zip(got[:2], alone[:2]))
        _check(_run(h, rows, pol, target, ref, smoothing=0.1, in_place=True), want, rows, 0.1, dtype, per_row)
    finally:
        a2t.a2t_prefer_destroy(h)


def test_captured(gpu):
    """Long and short answers' calls of one handle in a graph, replayed on new logits between eager calls."""
    import torch
    import paper_2609_31224_amd as a2t
    rng, vocab = np.random.default_rng(1), 100
    calls = [[300, 217], [5, 9]]
    pol, _ = _logits(rng, 517, vocab, "bf16")
    ref, _ = _logits(rng, 517, vocab, "bf16")
    _, target = _targets(rng, 517, vocab)
    side = torch.cuda.Stream()
    h, other = _handle(517, vocab, "bf16", stream=side), _handle(517, vocab, "bf16")
    outs = [(torch.zeros(3, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros_like(pol)) for _ in calls]
    try:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            for rows, (losses, ratios, grad) in zip(calls, outs):
                n = sum(rows)
                a2t.a2t_prefer_loss(h, rows, pol[:n], target[:n], losses, ref[:n], ratios=ratios, grad=grad[:n])
        for turn in range(3):
            pol[:, :vocab] = torch.randn((517, vocab), device="cuda")
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
            for rows, out in zip(calls, outs):
                n = sum(rows)
                want = _run(other, rows, pol[:n], target[:n], ref[:n])
                for x, y in zip(out, want[:3]):
                    assert np.array_equal(x[:len(y)].cpu().double().numpy(), y), turn
    finally:
        a2t.a2t_prefer_destroy(h)
        a2t.a2t_prefer_destroy(other)


def test_time_grows_with_the_rows(gpu):
    """Two answers of 2^18 rows: what every workgroup walked for itself would be 2^37 rows' statistics,
    seconds of them; formed once, the call takes milliseconds."""
    import torch
    import paper_2609_31224_amd as a2t
    n = 2 ** 18
    pol = torch.randn((2 * n, 8), device="cuda", dtype=torch.bfloat16)
    target = torch.zeros(2 * n, dtype=torch.int32, device="cuda")
    lp = torch.log_softmax(pol.float(), -1)[:, 0].contiguous()
    lp[n:] += 2.0 ** -14
    losses, ratios, grad = torch.zeros(3, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros_like(pol)
    h = _handle(2 * n, 8, "bf16")
    try:
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        a2t.a2t_prefer_loss(h, [n, n], pol, target, losses, ref_logp=lp, ratios=ratios, grad=grad)
        end.record()
        torch.cuda.synchronize()
        assert begin.elapsed_time(end) < 250.0
        # a row's ratio is off by 2^-20 and half a step of a log probability of at most 16, on both sides
        assert abs(float(ratios[0])) <= n * 2.0 ** -18 and abs(float(ratios[1]) + n * 2.0 ** -14) <= n * 2.0 ** -18
    finally:
        a2t.a2t_prefer_destroy(h)
