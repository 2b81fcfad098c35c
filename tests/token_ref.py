"""The calls on rows of token logits in float64, from their definitions, one row at a time on
the CPU, and what their 32-bit results may be off by.

EPS bounds the relative error that a result of 32-bit sums gathers per unit of what it is made
of: hardware exponentials and logarithms (2^-23), the rounding of their arguments (2^-24 of the
argument, which is why the span of the logits enters) and of sums of V numerators in at most some
hundred steps, whose errors mostly cancel: 32 units of 2^-22 for these, one for the argument."""
import math

import numpy as np

EPS = 2.0 ** -22
UNITS = 32.0
MIN_REST = 2.0 ** -20
# half a unit in the last place, relative, and the least difference near 0
# (numbers below the normal floats may be taken as 0 on the way)
ROUND = {"float32": (2.0 ** -24, 2.0 ** -125), "bfloat16": (2.0 ** -8, 2.0 ** -125),
         "float16": (2.0 ** -11, 2.0 ** -25)}


def span(row, T):
    """The range of a row's exponents, as far as 32-bit numerators are not 0."""
    row = row[np.isfinite(row)]
    return min(np.ptp(row) / T, 110.0) if row.size else 0.0


def lse(x):
    x = x[np.isfinite(x)]
    if not x.size:
        return -math.inf
    m = x.max()
    return m + math.log(np.exp(x - m).sum())


def top(row, K, T):
    order = np.lexsort((np.arange(row.size), -row))[:K]
    return row[order], order, lse(row / T)


def distill(row, values, indices, T, top_lse=None):
    """(loss, d loss / d row) of one row, each followed by the scale of its error: what it is
    made of, each part of relative error eps; a teacher's rest, 1 - sum p, is off by eps itself."""
    V = row.size
    if np.isfinite(row).any():
        row = row - row[np.isfinite(row)].max()    # q is the same, and rows of the lowest float have one
    keep = (indices >= 0) & (indices < V)
    at, t = indices[keep], values[keep] / T
    zero = np.zeros(V)
    if top_lse is None:
        p = np.exp(t - lse(t)) if np.isfinite(t).any() else np.zeros(t.size)
    elif top_lse == -math.inf:
        at, p = at[:0], t[:0]
    else:
        p = np.exp(t - top_lse)
    L = lse(row / T)
    dense = zero.copy()
    dense[at] = p
    if L == -math.inf:
        return (math.inf if (p > 0).any() else 0.0), 1.0, zero, zero
    logq = row / T - L
    q = np.exp(logq)
    on = dense > 0
    with np.errstate(divide="ignore", invalid="ignore"):
        loss = float((dense[on] * (np.log(dense[on]) - logq[on])).sum())
    if top_lse is None:
        if not on.any():
            return 0.0, 0.0, zero, zero
        return loss, 1 + abs(loss), (q - dense) / T, (q + dense) / T
    rest = np.ones(V, bool)
    rest[at] = False
    p_r = 1.0 - p.sum()
    if p_r <= MIN_REST:
        p_r = 0.0
    low = lse(row[rest] / T)
    scale = 1 + abs(loss)
    if p_r > 0:
        loss += p_r * (math.log(p_r) - (low - L))
        scale += abs(math.log(p_r) - (low - L))
    share = np.exp(row / T - low) if low > -math.inf else zero
    q_r = math.exp(low - L)
    grad = np.where(rest, share * (q_r - p_r), q - dense) / T
    return loss, scale, grad, np.where(rest, share * (q_r + p_r + 1), q + dense) / T


def verify(target, draft, tokens, uniforms, noise, n, T, draft_T, draft_lse=None):
    """(emitted, accepted, log-probabilities, margin) of one sequence; the margin is the least
    relative distance of a decision from going the other way."""
    V = target.shape[1]
    margin = math.inf

    def probs(row, T, L=None):
        L = lse(row / T) if L is None else L
        return np.exp(row / T - L) if L > -math.inf else np.zeros(V)

    a = 0
    while a < n:
        p = probs(target[a], T)
        q = probs(draft[a], draft_T, None if draft_lse is None else draft_lse[a])
        z = tokens[a]
        if not 0 <= z < V:
            break
        if p[z] > 0 and q[z] > 0:
            margin = min(margin, abs(uniforms[a] * q[z] - p[z]) / p[z])
        if not uniforms[a] * q[z] < p[z]:
            break
        a += 1
    p = probs(target[a], T)
    r = p
    if a < n:
        r = np.maximum(p - probs(draft[a], draft_T, None if draft_lse is None else draft_lse[a]), 0)
    if not (r > 0).any():
        r = p
    score = r / noise
    new = int(score.argmax())
    if score[new] > 0:
        others = np.delete(score, new)
        if others.size:
            margin = min(margin, 1 - others.max() / score[new])
    out = [int(z) for z in tokens[:a]] + [new]
    with np.errstate(divide="ignore"):
        logp = [float(np.log(probs(target[t], T)[z])) for t, z in enumerate(out)]
    return out, a, logp, margin
