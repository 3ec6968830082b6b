"""Causal attention over packed sequences, with gradients (oracle; test infrastructure only).

Plain float64 numpy, written from the definitions, one head at a time:

    O_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - lse_i),  lse_i = ln sum_j exp(scale q_i . k_j)

over the rows j of i's sequence with j <= i < until_j (every j <= i without ``until``); a row that
sees nothing has O = 0, lse = -inf and no gradient.  With delta_i = dO_i . O_i the gradients are

    dS_ij = p_ij (dO_i . v_j - delta_i),  dV_j = sum_i p_ij dO_i,
    dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i   (dK, dV: over a group's heads).

Query head h reads KV head h / (Hq / Hkv).  ``bounds`` turns half steps of the number types into
limits for every output, from the same sums with magnitudes in the place of values.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import Dict, Optional

import numpy as np


def visible(n: int, until: Optional[np.ndarray]) -> np.ndarray:
    """[n][n]: whether place i (row) sees place j (column)."""
    i = np.arange(n)
    see = i[None, :] <= i[:, None]
    if until is not None:
        see &= i[:, None] < np.asarray(until, np.int64)[None, :]
    return see


@dataclass
class PromptResult:
    o: np.ndarray                    # [rows][Hq][D]
    lse: np.ndarray                  # [Hq][rows]
    grads: Dict[str, np.ndarray] = field(default_factory=dict)    # dq, dk, dv
    bounds: Dict[str, np.ndarray] = field(default_factory=dict)   # how far each output may be off


def prompt_attention(seq_rows, q, k, v, until=None, d_o=None, scale=None, u_store: float = 0.0, u_mul: float = 0.0,
                     delta_rows: int = 0) -> PromptResult:
    """``u_store``: half a step of the type that outputs (and O, before the gradient reads it) are
    rounded to; ``u_mul``: of the type that probabilities and score gradients are rounded to before
    their products.  fp32 is assumed elsewhere.  Sequences of up to ``delta_rows`` rows have their
    delta as a sum of p_ij dO_i . v_j in fp32 instead of from the stored O."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    rows, hq, d = q.shape
    G = hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    e = 2.0 ** -24
    o, lse = np.zeros((rows, hq, d)), np.full((hq, rows), -np.inf)
    b_o, b_lse = np.zeros_like(o), np.zeros_like(lse)
    g = {c: np.zeros(x.shape) for c, x in (("dq", q), ("dk", k), ("dv", v))}
    b = {c: np.zeros(x.shape) for c, x in (("dq", q), ("dk", k), ("dv", v))}
    if d_o is not None:
        d_o = np.asarray(d_o, np.float64)
    at = 0
    for n in map(int, seq_rows):
        w = slice(at, at + n)
        see = visible(n, None if until is None else np.asarray(until)[w])
        has = see.any(1)
        at += n
        for h in range(hq):
            Q, K, V = q[w, h], k[w, h // G], v[w, h // G]
            s = np.where(see, scale * (Q @ K.T), -np.inf)
            top = np.where(has, s.max(1, initial=-np.inf), 0.0)
            z = np.exp(s - top[:, None]).sum(1)
            ls = np.where(has, top + np.log(np.where(has, z, 1.0)), -np.inf)
            p = np.exp(s - np.where(has, ls, 0.0)[:, None])
            O = p @ V
            o[w, h], lse[h, w] = O, ls
            # a score is a sum of d fp32 products, its exponential's argument a rounded difference of
            # numbers of its size; a probability is off by rho of itself
            size = np.abs(scale) * (np.abs(Q) @ np.abs(K).T)
            size = np.where(see, size, 0.0).max(1, initial=0.0)
            fl = np.where(has, np.abs(ls), 0.0)
            rho = (e * ((d + 8) * size + 8 * fl + 16))[:, None]
            sums = e * (n + 8)                    # fp32 sums over the keys (or queries)
            A = p @ np.abs(V)
            to = (2 * rho + u_mul + 2 * sums) * A + u_store * np.abs(O)
            b_o[w, h], b_lse[h, w] = to, (rho[:, 0] + sums) + 4 * e * (fl + size)
            if d_o is None:
                continue
            dO = d_o[w, h]
            dp = dO @ V.T
            delta = (dO * O).sum(1, keepdims=True)
            ds = p * (dp - delta)
            g["dq"][w, h] = scale * (ds @ K)
            g["dk"][w, h // G] += scale * (ds.T @ Q)
            g["dv"][w, h // G] += p.T @ dO
            # delta comes from the O that was stored; dO . v and delta are fp32 sums
            t = (np.abs(dO) * (to + u_store * to)).sum(1, keepdims=True)
            adp, adl = np.abs(dO) @ np.abs(V).T, (np.abs(dO) * np.abs(O)).sum(1, keepdims=True)
            if n <= delta_rows:
                t = (rho + e * (n + d + 16)) * (p * adp).sum(1, keepdims=True)
            off = p * (t + e * (d + 8) * (adp + adl)) + np.abs(ds) * (rho + u_mul + 2 * e)
            off_p = p * (rho + u_mul)
            abs_ds = p * (adp + adl)
            b["dq"][w, h] = scale * ((off + sums * abs_ds) @ np.abs(K))
            more = e * (G * n + 8)                # sums over the queries of all heads of the group
            b["dk"][w, h // G] += scale * ((off + more * abs_ds).T @ np.abs(Q))
            b["dv"][w, h // G] += (off_p + more * p).T @ np.abs(dO)
    out = PromptResult(o=o, lse=lse, bounds=dict(o=b_o, lse=b_lse))
    if d_o is not None:
        out.grads = g
        for c in g:
            b[c] += u_store * (np.abs(g[c]) + b[c])
        out.bounds.update(b)
    return out
