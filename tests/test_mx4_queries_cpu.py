"""CPU tests of what attention on an A2T_MX4 cache makes of its queries: three e2m3 numbers an
element hold what queries of uneven channels need, two do not, and the oracle's bound tells them apart."""
import numpy as np
import pytest

from oracle import mx4, rope
from oracle.attention import attend
from synth.streams import bf16_round

STEPS = (0, 4, 9)   # the parts' scales: 2^-step of the block's


def e2m3(x):
    """The nearest e2m3 number: steps of 1/8 below 2, 1/4 below 4, 1/2 up to 7.5."""
    a = np.abs(x)
    step = np.where(a < 2, 0.125, np.where(a < 4, 0.25, 0.5))
    return np.sign(x) * np.minimum(np.round(a / step) * step, 7.5)


def as_parts(x, steps):
    """``x[..., D]`` as the sum of one e2m3 number for each step, in units of a power of two for each 32
    elements of which the largest magnitude becomes 3.875 to 7.75."""
    y = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, mx4.BLOCK))
    a = np.abs(y).max(-1, keepdims=True)
    f = np.floor(np.log2(a))
    unit = np.ldexp(1.0, (f - 2 + (a >= 1.9375 * np.ldexp(1.0, f.astype(int)))).astype(int))
    out = np.zeros_like(y)
    for s in steps:
        out += e2m3((y - out) / unit * 2.0 ** s) * unit / 2.0 ** s
    return out.reshape(x.shape), np.broadcast_to(unit, y.shape).reshape(x.shape)


@pytest.mark.parametrize("spread", [1.0, 50.0, 1000.0])
def test_error_of_the_parts(spread):
    """1/4, 1/128 and 1/4096 unit, reached within a few per cent; a unit is 1/7.75 to 1/3.875 of the largest magnitude."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4000, 64))
    x[:, ::13] *= spread
    for n, most in ((1, 1 / 4), (2, 1 / 128), (3, 1 / 4096)):
        got, unit = as_parts(x, STEPS[:n])
        off = np.abs(got - x) / unit
        assert 0.9 * most < off.max() <= most
    top = np.abs(x / unit).reshape(-1, 32).max(-1)
    assert top.min() >= 3.875 and top.max() < 7.75


def uneven(rng, n, n_q, hq, hkv, d, q_spread, k_spread):
    """K, V of n rows and Q of the last n_q of them whose channels differ in size, four of Q's and others of K's standing
    out; K is scaled so that scores are spread by about 2.5, neither all alike nor one-hot."""
    k, v = (rng.standard_normal((n, hkv, d)) for _ in range(2))
    q = rng.standard_normal((n_q, hq, d))
    k[..., 5:d // 2:17] *= k_spread
    q[..., 3:d // 2:20] *= q_spread
    half = d // 2
    pairs = lambda x: np.square(x[..., :half]) + np.square(x[..., half:])   # noqa: E731
    spread = np.sqrt((pairs(q).mean((0, 1)) * pairs(k).mean((0, 1))).sum() / 2 / d)
    return bf16_round(k * 2.5 / spread), bf16_round(v), bf16_round(q)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_spread,k_spread", [(20.0, 20.0), (50.0, 20.0), (100.0, 50.0)])
def test_the_bound_tells_two_parts_from_three(d, q_spread, k_spread):
    rng = np.random.default_rng(2)
    n, n_q = 600, 16
    k, v, q = uneven(rng, n, n_q, 2, 1, d, q_spread, k_spread)
    c = mx4.OracleMx4Cache(2, 1, d, [0], theta=1e6)
    c.append(np.ones(n, np.uint8), np.arange(n), 0, {0: k}, {0: v})
    want, bound = c.attention_bound(0, q, n_q)
    pos = c.pos[-n_q:]
    turned = rope.rotate(q, pos, 1e6)

    def off(held):
        return np.abs(attend(held, c.k[0], c.v[0], pos, c.pos, c.scale) - want)
    two, three = (off(as_parts(turned, STEPS[:n])[0]) for n in (2, 3))
    assert (three / bound).max() <= 0.5 and (two / bound).max() > 1.5
    # queries rounded to bfloat16, as the bfloat16 caches' are, lie between them
    assert three.mean() < off(bf16_round(turned)).mean() < two.mean()
