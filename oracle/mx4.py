"""Rows held in 4 bits, float64 (oracle; test infrastructure only).

A head's row is cut into blocks of 32 elements.  Block scale 2^e: with a the block's largest
magnitude, e = floor(log2 a) - 2, and one more where a >= 1.75 * 2^floor(log2 a), kept within
[-124, 125].  Elements: the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (times 2^e, with a sign),
halfway cases to the one with the even place in that list, what lies beyond 6 to 6.  A
block with an infinity or a NaN is NaN throughout.

K is rotated before it is held: cosines and sines are those of 64 bits rounded to float32, the
products and their difference are exact to 64 bits, and the result is rounded to float32 once.
"""
from __future__ import annotations

import numpy as np

from . import rope
from .attention import attend
from .cache import OracleCache

BLOCK = 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E_MIN, E_MAX = -124, 125


def block_exponents(x: np.ndarray) -> np.ndarray:
    """e of every block of ``x[..., D]`` -> int [..., D / 32] (blocks of finite values)."""
    y = np.abs(np.asarray(x, np.float64)).reshape(x.shape[:-1] + (-1, BLOCK))
    a = y.max(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        f = np.floor(np.log2(a))
    f = np.where(a > 0, f, -1000)
    # log2 may round up to an integer just below a power of two
    f = np.where(np.ldexp(1.0, f.astype(int)) > a, f - 1, f).astype(int)
    e = f - 2 + (a >= 1.75 * np.ldexp(1.0, f))
    return np.clip(e, E_MIN, E_MAX)


def hold(x: np.ndarray) -> np.ndarray:
    """The values that rows ``x[..., D]`` are held as (float64)."""
    x = np.asarray(x, np.float64)
    y = x.reshape(x.shape[:-1] + (-1, BLOCK))
    bad = ~np.isfinite(y).all(-1, keepdims=True)
    z = np.where(bad, 0.0, y)
    s = np.ldexp(1.0, block_exponents(z.reshape(x.shape)))[..., None]
    t = np.abs(z) / s
    d = np.abs(t[..., None] - LEVELS)
    best = d.min(-1, keepdims=True)
    # of the (at most two) nearest levels the one with the even place
    place = np.arange(8)
    pick = np.argmin(np.where(d == best, place % 2 * 10, 100), -1)
    out = np.where(bad, np.nan, np.sign(z) * LEVELS[pick] * s)
    return out.reshape(x.shape)


def rotate_to_f32(x: np.ndarray, pos: np.ndarray, theta: float) -> np.ndarray:
    """``x[n][H][D]`` rotated by ``pos[n]``, rounded to float32 (returned as float64)."""
    x = np.asarray(x, np.float64)
    half = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None, None] * rope.inverse_frequencies(x.shape[-1], theta)
    c, s = (f(ang).astype(np.float32).astype(np.float64) for f in (np.cos, np.sin))
    lo, hi = x[..., :half], x[..., half:]
    with np.errstate(over="ignore", invalid="ignore"):
        return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1).astype(np.float32).astype(np.float64)


class OracleMx4Cache(OracleCache):
    """One stream's resident cache whose rows are held in 4 bits."""

    def append(self, seg, pos, unit, k=None, v=None):
        super().append(seg, pos, unit, k, v)
        n = self.step_rows
        for l in self.layers:
            self.k[l][-n:] = hold(rotate_to_f32(k[l], pos, self.theta))
            self.v[l][-n:] = hold(v[l])

    def attention_bound(self, layer, q, n_q, least=1e-6):
        """(o, bound): attention as OracleCache.attention's, and what a computation may be off by
        that holds rotated queries as three e2m3 numbers (an error of up to 1/4096 unit, the largest
        magnitude of a block of 32 being at least 3.875 units; independent from element to
        element), probabilities to 11 significant bits or 2^-25 of the largest, partial outputs to 11
        and the output to 8; `least`: and that partial outputs are fp16.

        A score's error is a sum of D independent ones, uniform in +- a_b |k_i| / (4096 * 3.875), a_b the
        largest magnitude of the query's block: six of its standard deviations are taken as its
        bound.  Besides, fp32 roundings of the rotation (four of 2^-24 of |x_i| + |x_{i+D/2}|), of the score's
        sum and of its difference to the reference (twelve of 2^-24 of the sum of magnitudes): 2^-20 of
        sum |k_i| (|x_i| + |x_{i+D/2}|).  An error d_j of the scores moves the output by p_j d_j (v_j - o) to first order,
        an error e_j of a probability by e_j (v_j - o); fp32 sums and exponentials take as much as
        2^-13 of the sum of magnitudes."""
        q_pos = self.pos[self.resident - n_q:]
        q_rot = rope.rotate(np.asarray(q, np.float64), q_pos, self.theta)
        k, v = self.k[layer], self.v[layer]
        o = attend(q_rot, k, v, q_pos, self.pos, self.scale)
        bound = np.zeros_like(o)
        G = self.Hq // self.Hkv
        mask = self.pos[None, :] <= q_pos[:, None]
        both = np.abs(np.asarray(q, np.float64))
        both = both + np.roll(both, both.shape[-1] // 2, -1)
        for h in range(self.Hq):
            kk, vv = k[:, h // G], v[:, h // G]
            s = np.where(mask, self.scale * (q_rot[:, h] @ kk.T), -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            most = np.repeat(np.abs(q_rot[:, h]).reshape(n_q, -1, BLOCK).max(-1), BLOCK, -1)
            d = 6 * self.scale / (4096 * 3.875 * np.sqrt(3)) * np.sqrt(np.square(most) @ np.square(kk).T)
            d += 2.0 ** -20 * self.scale * (both[:, h] @ np.abs(kk).T)
            for i in range(n_q):
                w = p[i] * d[i]
                e = np.where(mask[i], np.maximum(2.0 ** -11 * p[i], 2.0 ** -25 * p[i].max()), 0.0)
                bound[i, h] = np.abs(vv - o[i, h]).T @ (w + e) + 2.0 ** -13 * (np.abs(vv).T @ p[i])
        return o, bound + (2.0 ** -8 + 2.0 ** -11) * np.abs(o) + least
