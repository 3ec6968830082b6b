"""Scores that fp32 holds as -infinity, in every kind of workgroup of attention on A2T_MX4 caches: such a key has no
weight, and the keys behind it keep theirs, also where a wave's first keys are all of that kind."""
import numpy as np
import pytest

from oracle import mx4
from synth.streams import SEG_ACOUSTIC, bf16_round
from tests.test_gpu_mx4_shapes import NAMES, force

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("offset", [0.0, -60.0])   # of the other keys' scores
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", list(NAMES))
def test_keys_of_no_weight_come_first(gpu, monkeypatch, rows, d, offset, splits):
    """Keys 0 to 299 and 512 to 699 score -2^134 / sqrt(D), so that the first and later blocks of every wave hold nothing else;
    the others have scores of their own, all of them far below 0 or not."""
    import torch
    import paper_2609_31224_amd as a2t
    force(monkeypatch, rows, splits)
    rng = np.random.default_rng(5)
    hq, hkv, old, new, half = 4, 1, 1000, 20, d // 2
    n = old + new
    # the rotation by theta = 1e12 leaves the last dims of each half as they are
    k, q, v = np.zeros((n, hkv, d)), np.zeros((new, hq, d)), rng.standard_normal((n, hkv, d))
    dims = np.arange(d - 8, d - 2)
    k[..., dims], q[..., dims] = 4 * rng.standard_normal((n, hkv, 6)), 4 * rng.standard_normal((new, hq, 6)) / 4
    k[..., d - 2], q[..., d - 2] = 8.0, offset * np.sqrt(d) / 8
    none = np.r_[0:300, 512:700]
    k[none, :, half - 1] = -2.0 ** 120
    q[..., half - 1] = 2.0 ** 14
    k, q, v = bf16_round(k), bf16_round(q), bf16_round(v)
    kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16() for x in (k, v, q))
    seg = np.full(n, SEG_ACOUSTIC, np.uint8)
    c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, n, 0, old, rope_theta=1e12)
    o = torch.full_like(qd, float("nan"))
    a2t.a2t_append(c, 0, [0], [old], kd[:old], vd[:old], seg[:old], np.arange(old), [0])
    a2t.a2t_append_attn(c, 0, [0], [new], kd[old:], vd[old:], seg[old:], np.arange(old, n), [1], [new], qd, o)
    a2t.a2t_sync(c)
    a2t.a2t_cache_destroy(c)
    ref = mx4.OracleMx4Cache(hq, hkv, d, [0], theta=1e12)
    for unit, part in enumerate((slice(0, old), slice(old, n))):
        ref.append(seg[part], np.arange(n)[part], unit, {0: k[part]}, {0: v[part]})
    # the bound's score errors are those of keys that have a weight
    want, bound = ref.attention_bound(0, q, new)
    got = o.float().cpu().numpy().astype(np.float64)
    print(f"worst error {(np.abs(got - want) / bound).max():.3f} of its bound, bound {bound.max():.3f}", flush=True)
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("below", [12.5, 15.5, 18.5])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", list(NAMES))
def test_many_small_probabilities(gpu, monkeypatch, rows, d, below):
    """Every wave has one key of large score, whose value is 0, and many others at 2^-below of its probability: as
    fp16 numbers these are normal or subnormal, and products and sums both have to count them."""
    import torch
    import paper_2609_31224_amd as a2t
    force(monkeypatch, rows, 1)
    rng = np.random.default_rng(6)
    hq, hkv, old, new = 4, 1, 4000, 33
    n = old + new
    k, q, v = np.zeros((n, hkv, d)), np.zeros((new, hq, d)), 8 + rng.random((n, hkv, d))
    peaks = np.arange(0, 256, 32)
    k[peaks, :, d - 1] = 4.0
    v[peaks] = 0.0
    q[..., d - 1] = below * np.log(2) * np.sqrt(d) / 4     # theta = 1e12 leaves the last dim as it is
    k, q, v = bf16_round(k), bf16_round(q), bf16_round(v)
    kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16() for x in (k, v, q))
    seg = np.full(n, SEG_ACOUSTIC, np.uint8)
    c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, n, 0, 1024, rope_theta=1e12)
    ref = mx4.OracleMx4Cache(hq, hkv, d, [0], theta=1e12)
    o = torch.full_like(qd, float("nan"))
    for unit, at in enumerate((0, 1000, 2000, 3000, old)):
        part = slice(at, min(at + 1000, old) if at < old else n)
        m = part.stop - part.start
        ref.append(seg[part], np.arange(n)[part], unit, {0: k[part]}, {0: v[part]})
        if at < old:
            a2t.a2t_append(c, 0, [0], [m], kd[part], vd[part], seg[part], np.arange(n)[part], [unit])
        else:
            a2t.a2t_append_attn(c, 0, [0], [m], kd[part], vd[part], seg[part], np.arange(n)[part], [unit], [m], qd, o)
    a2t.a2t_sync(c)
    a2t.a2t_cache_destroy(c)
    want, bound = ref.attention_bound(0, q, new, least=0.0)
    got = o.float().cpu().numpy().astype(np.float64)
    print(f"worst error {(np.abs(got - want) / bound).max():.3f} of its bound, outputs {want.mean():.4f}, bound {bound.max():.5f}", flush=True)
    assert (np.abs(got - want) <= bound).all()
    # the small ones missing from the products, or (where they are a share of the sum worth it) from the sum, would
    # not be within the bound: without them in the sum outputs grow by that share of themselves
    share = want / 8.5
    assert (bound < want / 2).all() and ((bound < want * share).all() or below > 16)
