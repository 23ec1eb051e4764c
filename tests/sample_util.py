"""Tokens from logits in 64 bits, row by row, from the definition: used by the tests of npd_sample_tokens."""
import numpy as np


def draw(row, u, tau, top_k, top_p, min_p):
    """(token, kept, logprob, nll) of one row of finite logits and -inf (float64); None where there is nothing to draw from."""
    ids = np.flatnonzero(row > -np.inf)
    if not len(ids):
        return None
    ids = ids[np.argsort(-row[ids], kind="stable")]
    x = row[ids]
    nll = np.log(np.sum(np.exp(x - x[0]))) + (x[0] - x)
    if tau == 0:
        return int(ids[0]), 1, 0.0, float(nll[0])
    w = np.exp((x - x[0]) / tau)
    n = min(top_k, len(ids)) if top_k > 0 else len(ids)
    total = np.cumsum(w)
    if top_p < 1:
        n = min(n, int(np.count_nonzero(total < top_p * total[n - 1])) + 1)
    if min_p > 0:
        n = min(n, int(np.count_nonzero(w >= min_p)))
    n = max(n, 1)
    j = min(int(np.count_nonzero(total[:n] <= u * total[n - 1])), n - 1)
    return int(ids[j]), n, float(np.log(w[j] / total[n - 1])), float(nll[j])
