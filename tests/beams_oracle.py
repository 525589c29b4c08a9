"""The choice of beams of include/lessdec.h written out in numpy and float64: what the tests compare with."""
import numpy as np


def select(x, score, ended, groups, beams, picks, end_token):
    """x float64 [rows, vocab]; parent, token, c (float64), ended of [groups, picks]."""
    vocab = x.shape[1]
    parent, token = np.full((groups, picks), -1), np.full((groups, picks), -1)
    best = np.full((groups, picks), -np.inf)
    for g in range(groups):
        c, beam, logit, v = [], [], [], []
        for b in range(beams):
            r = g * beams + b
            if ended is not None and ended[r]:
                row, logits, tokens = np.array([score[r]]), np.zeros(1), np.array([end_token])
            else:
                with np.errstate(all="ignore"):
                    top = x[r].max()
                    row = score[r] + (x[r] - (top + np.log(np.exp(x[r] - top).sum())))
                logits, tokens = x[r], np.arange(vocab)
            there = row > -np.inf                             # (false where it is NaN)
            c.append(row[there]); logit.append(logits[there]); v.append(tokens[there]); beam.append(np.full(there.sum(), b))
        c, beam, logit, v = (np.concatenate(p) for p in (c, beam, logit, v))
        order = np.lexsort((v, -logit, beam, -c))[:picks]
        n = len(order)
        parent[g, :n], token[g, :n], best[g, :n] = g * beams + beam[order], v[order], c[order]
    return parent, token, best, (parent >= 0) & (token == end_token)
