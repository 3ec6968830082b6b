"""The preference loss of paired answers on given logits (oracle; test infrastructure only): float64
numpy from the definition.  Answers 2p (chosen) and 2p + 1 (rejected) of pair p follow each other;
rows whose target is outside the vocabulary take no part."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import numpy as np


def log_softmax(x):
    x = np.asarray(x, np.float64)
    m = x.max(-1, keepdims=True)
    return x - m - np.log(np.exp(x - m).sum(-1, keepdims=True))


def token_logp(logits, target) -> np.ndarray:
    target = np.asarray(target)
    vocab = np.asarray(logits).shape[1]
    used = (target >= 0) & (target < vocab)
    lp = log_softmax(logits)
    return np.where(used, lp[np.arange(len(target)), np.where(used, target, 0)], 0.0)


@dataclass
class PreferResult:
    loss: float
    margin: float          # mean of h
    won: float             # share of pairs with h > 0
    ratios: np.ndarray     # [answers]
    slope: np.ndarray      # [rows] dL / d ln p_policy(target)
    grad: np.ndarray       # [rows][vocab]


def prefer_loss(answer_rows, policy, target, reference=None, ref_logp: Optional[np.ndarray] = None, beta: float = 0.1,
                smoothing: float = 0.0) -> PreferResult:
    target, rows = np.asarray(target), np.asarray(answer_rows, np.int64)
    n, vocab = np.asarray(policy).shape
    used = (target >= 0) & (target < vocab)
    ref = token_logp(reference, target) if reference is not None else np.where(used, np.asarray(ref_logp, np.float64), 0.0)
    diff = token_logp(policy, target) - ref
    answer = np.repeat(np.arange(len(rows)), rows)
    ratios = np.bincount(answer, diff, minlength=len(rows))
    h = beta * (ratios[0::2] - ratios[1::2])
    # a term without weight is left out, also where h is infinite (a target whose logit is -infinity)
    loss = sum((w * np.logaddexp(0, x) if w > 0 else np.zeros(len(h))) for w, x in ((1 - smoothing, -h), (smoothing, h))).mean()
    # d ln sigma(h) / dh = sigma(-h)
    with np.errstate(over="ignore"):
        up, down = 1 / (1 + np.exp(h)), 1 / (1 + np.exp(-h))
    c = -beta * ((1 - smoothing) * up - smoothing * down) / len(h)
    slope = np.where(used, np.stack([c, -c], -1).ravel()[answer], 0.0)
    grad = -slope[:, None] * np.exp(log_softmax(policy))
    grad[np.flatnonzero(used), target[used]] += slope[used]
    return PreferResult(loss=float(loss), margin=float(h.mean()), won=float((h > 0).mean()), ratios=ratios, slope=slope, grad=grad)
