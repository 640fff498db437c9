"""A plain model of beam search's selection in 64 bits: every candidate, sorted."""
import numpy as np


def select(logits, scores, ended, end_token, keep, most):
    """logits float64 [groups, beams, vocab], scores [groups, beams], ended bool or None; most: the largest finite value of
    the logits' type.  Returns scores (float64), tokens, parents, ended, as include/less.h says."""
    groups, beams, vocab = logits.shape
    x = np.where(np.isnan(logits), -np.inf, np.minimum(logits, most))
    out = (np.full((groups, keep), -np.inf), np.full((groups, keep), -1), np.zeros((groups, keep), int),
           np.zeros((groups, keep), bool))
    for g in range(groups):
        v = np.full((beams, vocab), -np.inf)
        for b in range(beams):
            if not np.isfinite(scores[g, b]):
                continue
            if ended is not None and ended[g, b]:
                v[b, end_token] = scores[g, b]
            elif x[g, b].max() > -np.inf:
                top = x[g, b].max()
                v[b] = scores[g, b] + (x[g, b] - (top + np.log(np.exp(x[g, b] - top).sum())))
        v = v.ravel()
        # equal values: the lowest beam, of one beam the larger logit (beside a very large one values lose it), the lowest token
        beam = np.repeat(np.arange(beams), vocab)
        order = np.lexsort((np.where(np.isnan(x[g]), -np.inf, -x[g]).ravel(), beam, -v))[:keep]
        for k in range(keep):
            some = k < len(order) and v[order[k]] > -np.inf
            out[2][g, k] = g * beams + (order[k] // vocab if some else min(k, beams - 1))
            if some:
                out[0][g, k], out[1][g, k] = v[order[k]], order[k] % vocab
                out[3][g, k] = out[1][g, k] == end_token
    return out
