"""One prompt, many continuations, in numpy from the definitions in include/attn.h: attention over a prefix and a sequence's own tokens, the choice
among beams, and which sequence a reordered one comes from."""
import numpy as np


def attend(q, prefix, own, n, alpha, causal):
    """As oracle.cache.attend (O, LSE, sum of P |v|) for the newest queries q of a sequence; prefix, own: (K, V) of its prefix and its own tokens;
    n: queries that are real (the first ones)."""
    d = q.shape[1]
    k, v = (np.concatenate(x) for x in zip(prefix, own))
    length, before = len(own[0]), len(prefix[0])
    O, lse, size = np.zeros((len(q), d)), np.full(len(q), -np.inf), np.zeros((len(q), d))
    for i in range(n):
        seen = before + (min(length, max(0, length - n + i + 1)) if causal else length)
        if seen == 0:
            continue
        s = alpha * (k[:seen] @ q[i])
        m = s.max()
        p = np.exp(s - m)
        lse[i] = m + np.log(p.sum())
        p /= p.sum()
        O[i], size[i] = p @ v[:seen], p @ np.abs(v[:seen])
    return O, lse, size


def select(logits, scores, n, finished=None, end_token=-1):
    """Of one item: parents, tokens, sums, ended; logits [beams, V] and scores [beams] in 64 bits."""
    found = []
    for k, (x, score) in enumerate(zip(np.asarray(logits, dtype=np.float64), np.asarray(scores, dtype=np.float64))):
        if not np.isfinite(score):
            continue
        if finished is not None and finished[k]:
            found.append((-score, k, 0.0, end_token, True))
            continue
        if np.isnan(x).any() or x.max() == np.inf or x.max() == -np.inf:
            continue
        m = x.max()
        total = score + (x - m) - np.log(np.exp(x - m).sum())
        at = np.flatnonzero(x > -np.inf)
        at = at[np.lexsort((at, -x[at]))][:n]              # (a beam gives n at most)
        found += [(-total[t], k, -x[t], int(t), t == end_token) for t in at]
    found.sort()
    found = found[:n]
    rest = n - len(found)
    return ([f[1] for f in found] + [-1] * rest, [f[3] for f in found] + [-1] * rest, [-f[0] for f in found] + [-np.inf] * rest,
            [bool(f[4]) for f in found] + [False] * rest)


def origin(parents):
    """Of one group: for each place the place whose sequence it gets."""
    return [p if 0 <= p < len(parents) else s for s, p in enumerate(parents)]
