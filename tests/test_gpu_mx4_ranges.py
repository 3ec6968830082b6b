"""Rows of A2T_MX4 caches whose scales are at the ends of their range, attended with one split: every output
element within a bound in proportion to the outputs, which zeros in their place would not meet."""
import numpy as np
import pytest

from oracle import mx4
from synth.streams import bf16_round
from tests.test_gpu_mx4_queries import attend_on
from tests.test_gpu_mx4_shapes import NAMES, force
from synth.streams import SEG_ACOUSTIC

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k_exp,q_exp,v_exp", [(-125, 123, -125), (-124, 100, -40), (126, -110, 100), (0, 0, -100), (100, -100, 110)])
@pytest.mark.parametrize("d,hq,hkv", [(64, 8, 2), (128, 4, 1)])
@pytest.mark.parametrize("rows", list(NAMES))
def test_scales_at_the_ends(gpu, monkeypatch, rows, d, hq, hkv, k_exp, q_exp, v_exp):
    force(monkeypatch, rows, 1)
    rng = np.random.default_rng(12)
    n, new = 400, 33
    big = 2.0 ** 127 * 1.9921875     # the largest bfloat16 number
    k, v, q = (bf16_round(np.clip(rng.standard_normal((m, h, d)) * 2.0 ** e, -big, big))
               for m, h, e in ((n, hkv, k_exp), (n, hkv, v_exp), (new, hq, q_exp)))
    ref = mx4.OracleMx4Cache(hq, hkv, d, [0], theta=1e6)
    ref.append(np.full(n, SEG_ACOUSTIC), np.arange(n), 0, {0: k}, {0: v})
    for x, e in ((ref.k[0], k_exp), (ref.v[0], v_exp)):
        # a block whose largest element lies just above 2^e has scale 2^(e - 2), one with twice that 2^(e - 1)
        held = mx4.block_exponents(x)
        assert held.min() == max(mx4.E_MIN, e - 2) or held.max() == min(mx4.E_MAX, e)
    got = attend_on(k, v, q, hq, hkv, d, new)
    # bfloat16 has steps of 2^-133 below 2^-126
    want, bound = ref.attention_bound(0, q, new, least=2.0 ** -133)
    off = np.abs(got - want) / bound
    assert np.isfinite(off).all()
    print(f"worst error {off.max():.3f} of its bound, zeros {(np.abs(want) / bound).max():.1f} of it", flush=True)
    assert off.max() <= 1.0
    assert (np.abs(want) / bound).max() > 8
