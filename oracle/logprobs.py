"""Oracle of a step's log probabilities (test infrastructure): 64 bits, from the
definitions."""
import math

import numpy as np


def logprobs(logits, tokens, top=0, temperature=1.0):
    """logits [R, V] (float), tokens [R]: log probabilities, entropies, and the `top`
    largest logits' indices (-1: none) and log probabilities."""
    R, V = logits.shape
    lp, ent = np.full(R, np.nan), np.full(R, np.nan)
    ids, alt = np.full((R, top), -1, np.int64), np.full((R, top), np.nan)
    for r in range(R):
        x = logits[r].astype(np.float64) / temperature
        order = np.lexsort((np.arange(V), -logits[r].astype(np.float64)))  # (NaN last)
        best = [i for i in order[: top] if not np.isnan(x[i])]
        ids[r, : len(best)] = best
        if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
            continue
        m = int(order[0])
        d = x - x[m]
        e = np.exp(d)
        rest = math.fsum(np.delete(e, m))
        log_z = math.log1p(rest)
        t = int(tokens[r])
        lp[r] = d[t] - log_z if 0 <= t < V else -np.inf
        seen = e > 0
        ent[r] = log_z - math.fsum(e[seen] * d[seen]) / (1 + rest)
        alt[r, : len(best)] = d[best] - log_z
    return lp, ent, ids, alt
