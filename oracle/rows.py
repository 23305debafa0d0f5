"""Operators on rows of logits in float64: sampling, token log-probabilities, GRPO's policy loss, distillation.

Rows are float64 arrays [rows][vocab] of the values that the inputs hold. -inf is a token that cannot occur; a row
without a finite logit is empty (token -1, log-probability -inf, entropy, loss and gradient 0); NaN or +inf makes a
row's token -1 and its other results NaN. Each function goes through its rows one by one from the definition.
"""
import math

import numpy as np

TAIL = 2.0 ** -24


def row_state(x):
    """"ok", "empty" or "bad"."""
    if np.isnan(x).any() or (x == np.inf).any():
        return "bad"
    return "ok" if (x > -np.inf).any() else "empty"


def log_softmax(x, temperature=1.0):
    z = (x - x.max()) / temperature
    return z - math.log(math.fsum(np.exp(z)))


def log_sum(logs):
    """ln of the sum of exp(logs); -inf where none is finite."""
    if not (logs > -np.inf).any():
        return -math.inf
    top = logs.max()
    return top + math.log(math.fsum(np.exp(logs - top)))


def _entropy(lp):
    seen = lp[lp > -np.inf]
    return -math.fsum(np.exp(seen) * seen)


def kept_tokens(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Indices of the tokens that are kept, the likeliest first (the lowest index among equals)."""
    order = np.argsort(-x, kind="stable")
    with np.errstate(invalid="ignore"):
        w = np.where(x > -np.inf, np.exp((x - x.max()) / temperature), 0.0)[order]
    n = len(x)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        want = max(top_p, 0.0) * math.fsum(w[:n])
        sums = np.cumsum(w[:n])
        n = 1 + int((sums[:-1] < want).sum())
    if min_p > 0:
        n = min(n, int((w >= min(min_p, 1.0)).sum()))
    return order[:max(n, 1)]


def _at(a, n, default):
    return default if a is None else a[n].item()


def sample(x, u, *, temperature=None, top_k=None, top_p=None, min_p=None):
    """tokens, logprobs, kept_logprobs, and each row's distance of u from the nearest border of its token's interval."""
    tokens, logprobs, kept, margin = [], [], [], []
    for n, row in enumerate(x):
        state = row_state(row)
        if state != "ok":
            tokens.append(-1)
            logprobs.append(-math.inf if state == "empty" else math.nan)
            kept.append(logprobs[-1])
            margin.append(math.inf)
            continue
        T = _at(temperature, n, 1.0)
        if not T > 0:
            tokens.append(int(row.argmax()))
            logprobs.append(log_softmax(row)[tokens[-1]])
            kept.append(0.0)
            margin.append(math.inf)
            continue
        p = _at(top_p, n, 1.0)
        q = _at(min_p, n, 0.0)
        ids = np.sort(kept_tokens(row, T, _at(top_k, n, 0), 1.0 if math.isnan(p) else p, 0.0 if math.isnan(q) else q))
        with np.errstate(invalid="ignore"):
            w = np.where(row[ids] > -np.inf, np.exp((row[ids] - row.max()) / T), 0.0)
        total = math.fsum(w)
        sums = np.cumsum(w) / total
        at = _at(u, n, 0.0)
        at = 0.0 if math.isnan(at) else min(max(at, 0.0), 1 - 2.0 ** -24)
        i = min(int(np.searchsorted(sums, at, side="right")), len(ids) - 1)
        tokens.append(int(ids[i]))
        lp = log_softmax(row, T) if math.isfinite(T) else np.where(row > -np.inf, -math.log((row > -np.inf).sum()), -np.inf)
        logprobs.append(lp[ids[i]])
        kept.append(math.log(w[i] / total))
        margin.append(min(abs(sums[i] - at), abs(at - sums[i - 1]) if i and at > 0 else math.inf))
    return np.array(tokens), np.array(logprobs), np.array(kept), np.array(margin)


def token_logprobs(x, tokens, temperature=1.0):
    n = len(x)
    lp, H = np.zeros(n), np.zeros(n)
    for r, row in enumerate(x):
        if not 0 <= tokens[r] < x.shape[1]:
            continue
        state = row_state(row)
        if state == "ok":
            l = log_softmax(row, temperature)
            lp[r], H[r] = l[tokens[r]], _entropy(l)
        else:
            lp[r], H[r] = (-np.inf, 0.0) if state == "empty" else (np.nan, np.nan)
    return lp, H


@np.errstate(over="ignore")
def policy_loss(x, tokens, old, advantages, *, row_seq=None, weights=None, ref=None, temperature=1.0, clip_low=0.2,
                clip_high=0.2, kl_beta=0.0, entropy_coef=0.0):
    """losses, logprobs, entropy, dlogits."""
    n, V = x.shape
    adv = np.asarray(advantages, np.float64).reshape(-1)
    loss, grad = np.zeros(n), np.zeros((n, V))
    seq = np.arange(n) if row_seq is None else np.asarray(row_seq)
    known = (seq >= 0) & (seq < len(adv))
    lp, H = token_logprobs(x, np.where(known, tokens, -1), temperature)
    for r in range(n):
        y, w = int(tokens[r]), 1.0 if weights is None else float(weights[r])
        if not (0 <= y < V and known[r]) or w == 0 or row_state(x[r]) == "empty":
            continue
        if row_state(x[r]) == "bad":
            loss[r], grad[r] = np.nan, np.nan
            continue
        l, A = log_softmax(x[r], temperature), adv[seq[r]]
        p = np.exp(l)
        # r of a token that cannot occur is 0; an advantage of 0 has no surrogate, however large r is.
        ratio = 0.0 if l[y] == -np.inf else min(float(np.exp(l[y] - old[r])), np.finfo(np.float64).max)
        free, held = ratio * A, min(max(ratio, 1 - clip_low), 1 + clip_high) * A
        value, g = -min(free, held) - entropy_coef * H[r], -free if free <= held else 0.0
        if kl_beta:
            gap = ref[r] - l[y]
            value += kl_beta * (math.exp(gap) - gap - 1)
            g += kl_beta * (1 - math.exp(gap))
        loss[r] = w * value
        d = -g * p + entropy_coef * p * (np.where(p > 0, l, 0.0) + H[r])
        d[y] += g
        grad[r] = w / temperature * d
    return loss, lp, H, grad


@np.errstate(invalid="ignore", over="ignore")
def distill_loss(x, ids, values, *, kind="tail", weights=None, temperature=1.0):
    """losses, dlogits."""
    n, V = x.shape
    loss, grad = np.zeros(n), np.zeros((n, V))
    for r in range(n):
        w, state = 1.0 if weights is None else float(weights[r]), row_state(x[r])
        if w == 0 or state == "empty":
            continue
        if state == "bad":
            loss[r], grad[r] = np.nan, np.nan
            continue
        entries = {}
        for i, t in zip(ids[r].tolist(), values[r].astype(np.float64).tolist()):
            if 0 <= i < V and t != -math.inf:
                entries.setdefault(i, t)
        at = np.array(list(entries), int)
        t = np.array(list(entries.values()), np.float64)
        l = log_softmax(x[r], temperature)
        q, lq = np.exp(l), l[at]
        if kind == "topk":
            if not len(at):
                continue
            t = t / temperature
            t = t - t.max()
            lp = t - math.log(math.fsum(np.exp(t)))
            P = np.exp(lp)
            value, d = math.fsum(np.where(P == 0, 0.0, P * (lp - lq))), q.copy()
            d[at] -= P
        else:
            P = np.exp(t)
            rest = max(1 - math.fsum(P), TAIL)
            others = np.ones(V, bool)
            others[at] = False
            # Where the mass outside is below float64's range it still has a logarithm.
            log_out = log_sum(l[others])
            outside, out = log_out > -math.inf, math.exp(log_out)
            gap = log_out - math.log(rest) if outside else 0.0
            if kind == "tail":
                value = math.fsum(np.where(P == 0, 0.0, P * (t - lq))) - (rest * gap if outside else 0.0)
                whole = math.fsum(P) + (rest if outside else 0.0)
                d = whole * q - rest * np.exp(np.where(others, l - log_out, -np.inf)) if outside else np.zeros(V)
                d[at] = whole * q[at] - P
            else:
                value = math.fsum(np.where(q[at] == 0, 0.0 * P, q[at] * (lq - t))) + out * gap
                d = q * (gap - value) if outside else np.zeros(V)
                d[at] = np.where(q[at] > 0, q[at] * (lq - t - value), 0.0)
        loss[r], grad[r] = w * value, w / temperature * d
    return loss, grad
