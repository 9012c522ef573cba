"""Layer norm, embedding and distillation by their definitions, in 64 bits (test infrastructure only)."""
import numpy as np


def norm_fwd(x, gamma, beta, eps):
    """(y, mean, rstd)"""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def norm_bwd(x, g, gamma, mean, rstd):
    """(g_x, g_gamma, g_beta) from given statistics"""
    x, g, mean, rstd = (np.asarray(a, dtype=np.float64) for a in (x, g, mean, rstd))
    xh = (x - mean[:, None]) * rstd[:, None]
    u = g * gamma
    g_x = rstd[:, None] * (u - u.mean(1, keepdims=True) - xh * (u * xh).mean(1, keepdims=True))
    return g_x, (g * xh).sum(0), g.sum(0)


def embed_fwd(tokens, table, scale, padding):
    """Rows of zeros for padding and for tokens outside the table"""
    table = np.asarray(table, dtype=np.float64)
    ok = (tokens != padding) & (tokens >= 0) & (tokens < len(table))
    return np.where(ok[:, None], table[np.where(ok, tokens, 0)] * scale, 0.0)


def embed_bwd(tokens, g, scale, padding, vocabulary):
    """(gradient of the table, sums of the magnitudes that make it up)"""
    g = np.asarray(g, dtype=np.float64)
    ok = (tokens != padding) & (tokens >= 0) & (tokens < vocabulary)
    out, mag = np.zeros((vocabulary, g.shape[1])), np.zeros((vocabulary, g.shape[1]))
    np.add.at(out, tokens[ok], g[ok] * scale)
    np.add.at(mag, tokens[ok], np.abs(g[ok] * scale))
    return out, mag


def token_order(tokens, padding, vocabulary):
    """(sorted tokens, positions): stable, padding and tokens outside the vocabulary last, as `vocabulary`"""
    ok = (tokens != padding) & (tokens >= 0) & (tokens < vocabulary)
    key = np.where(ok, tokens, vocabulary)
    index = np.argsort(key, kind="stable")
    return key[index], index


def _log_softmax(v):
    v = v - v.max()
    return v - np.log(np.exp(v).sum())


def distill(z, ids, logits, T, hard, labels, w):
    """(row losses, gradient): a row of weight 0, and an absent term, leave zeros"""
    z = np.asarray(z, dtype=np.float64)
    rows, classes = z.shape
    loss, g = np.zeros(rows), np.zeros((rows, classes))
    with np.errstate(all="ignore"):
        for r in range(rows):
            if w[r] == 0:
                continue
            t = np.asarray(logits[r], dtype=np.float64)
            ok = (ids[r] >= 0) & (ids[r] < classes) & ~np.isneginf(t)
            if ok.any() and hard < 1:
                lp, lq = _log_softmax(t[ok] / T), _log_softmax(z[r] / T)
                p = np.exp(lp)
                at = ids[r][ok]
                loss[r] += (1 - hard) * T * T * np.where(p == 0, 0.0, p * (lp - lq[at])).sum()
                d = np.exp(lq)
                np.add.at(d, at, -p)
                g[r] += w[r] * (1 - hard) * T * d
            y = -1 if labels is None else labels[r]
            if hard > 0 and 0 <= y < classes:
                lq = _log_softmax(z[r])
                loss[r] += hard * -lq[y]
                d = np.exp(lq)
                d[y] -= 1
                g[r] += w[r] * hard * d
    return loss, g
