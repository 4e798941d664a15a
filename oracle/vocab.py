"""Oracle of the vocabulary's two ends of a policy-gradient pass, in float64, from the definitions in include/rollout.h."""
import numpy as np


def _softmax(x, temperature):
    """(differences from the maximum over T, ln of the sum of their exponentials, probabilities) of one row; None for a
    row of -inf alone."""
    top = np.max(x)
    if top == -np.inf:
        return None
    d = (x - top) / temperature
    log_s = np.log(np.sum(np.exp(d)))
    return d, log_s, np.exp(d - log_s)


def _entropy(d, log_s, p):
    if np.isnan(log_s):
        return np.nan
    held = p > 0
    return -np.sum(p[held] * (d[held] - log_s))


def token_logprobs(x, targets, temperature, top=0):
    """logits [rows][vocab] -> logp, entropy, row_stats, top_ids, top_logp."""
    x = np.asarray(x, np.float64)
    rows, vocab = x.shape
    logp, entropy, stats = np.zeros(rows), np.zeros(rows), np.zeros((rows, 2))
    ids, alt = np.zeros((rows, top), np.int32), np.zeros((rows, top))
    for r in range(rows):
        t = -1 if targets is None else int(targets[r])
        has = 0 <= t < vocab
        if np.isnan(x[r]).any() or np.isposinf(x[r]).any():
            logp[r] = np.nan if has else 0.0
            entropy[r] = np.nan
            stats[r] = np.nan
            alt[r] = np.nan
        else:
            s = _softmax(x[r], temperature)
            if s is None:
                logp[r] = -np.inf if has else 0.0
                stats[r] = -np.inf
                alt[r] = -np.inf
            else:
                d, log_s, p = s
                logp[r] = d[t] - log_s if has else 0.0
                entropy[r] = _entropy(d, log_s, p)
                stats[r] = np.max(x[r]), log_s
        # greatest first, equal ones by ascending id, NaN last
        key = np.where(np.isnan(x[r]), -np.inf, x[r])
        ids[r] = np.lexsort((np.arange(vocab), -key, np.isnan(x[r])))[:top]
        if not np.isnan(alt[r]).any() and s is not None:
            alt[r] = d[ids[r]] - log_s
    return logp, entropy, stats, ids, alt


def token_logprobs_grad(x, targets, temperature, grad_logp, grad_entropy=None):
    """d/dx of sum grad_logp logp + grad_entropy entropy."""
    x = np.asarray(x, np.float64)
    out = np.zeros_like(x)
    for r in range(len(x)):
        t = -1 if targets is None else int(targets[r])
        g = float(grad_logp[r]) if 0 <= t < x.shape[1] else 0.0
        h = 0.0 if grad_entropy is None else float(grad_entropy[r])
        if g == 0.0 and h == 0.0:
            continue
        if np.isnan(x[r]).any() or np.isposinf(x[r]).any():
            out[r] = np.nan
            continue
        s = _softmax(x[r], temperature)
        if s is None:
            continue
        d, log_s, p = s
        held = p > 0
        out[r] = -g * p
        out[r][held] -= h * p[held] * (d[held] - log_s + _entropy(d, log_s, p))
        if g:
            out[r][t] += g
        out[r] /= temperature
    return out


def embed(table, tokens, scale):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for r, t in enumerate(tokens):
        if 0 <= t < len(table):
            out[r] = scale * table[t]
    return out


def embed_grad(grad_rows, tokens, vocab, scale, base=None):
    grad_rows = np.asarray(grad_rows, np.float64)
    out = np.zeros((vocab, grad_rows.shape[1]))
    for r, t in enumerate(tokens):
        if 0 <= t < vocab:
            out[t] += grad_rows[r]
    return scale * out + (0.0 if base is None else np.asarray(base, np.float64))


def head_logprobs(hidden, lm_head, targets, temperature):
    x = np.asarray(hidden, np.float64) @ np.asarray(lm_head, np.float64).T
    return token_logprobs(x, targets, temperature)[:3]


def head_logprobs_grad(hidden, lm_head, targets, temperature, grad_logp, grad_entropy=None):
    """(grad_hidden, grad_head, the logits' gradient)."""
    hidden, lm_head = np.asarray(hidden, np.float64), np.asarray(lm_head, np.float64)
    dx = token_logprobs_grad(hidden @ lm_head.T, targets, temperature, grad_logp, grad_entropy)
    return dx @ lm_head, dx.T @ hidden, dx
