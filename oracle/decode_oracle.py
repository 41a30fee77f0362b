"""Float64 statement of decoding over a compacted cache: attention of new tokens over a cache and a tree of themselves, the
attention weight of accepted tokens, commit and eviction.  One KV head of one sequence at a time, plain loops; shares no code with
the GPU path."""
import numpy as np


def visible(n, n_new, masks):
    """[n_new, n + n_new]: which slots a new token sees.  ``masks``: a word per new token, or None (those before it and itself)."""
    see = np.zeros((n_new, n + n_new), dtype=bool)
    see[:, :n] = True
    for i in range(n_new):
        for u in range(n_new):
            see[i, n + u] = u <= i if masks is None else bool(int(masks[i]) >> u & 1)
    return see


def attend(q, k, v, positions, n, scale, softcap=0.0, slopes=None, masks=None):
    """q [n_new, G, d] over k, v [n + n_new, d]: out [n_new, G, d], lse [n_new, G] and the probabilities [n_new, G, n + n_new].
    What a row does not see has no part in it."""
    t, g, d = q.shape
    see = visible(n, t, masks)
    out, lse = np.zeros((t, g, d)), np.full((t, g), -np.inf)
    p = np.zeros((t, g, n + t))
    for i in range(t):
        at = np.flatnonzero(see[i])
        if len(at) == 0:
            continue
        x = (q[i] @ k[at].T) * scale
        if softcap:
            x = softcap * np.tanh(x / softcap)
        if slopes is not None:
            x = x - np.asarray(slopes, dtype=np.float64)[:, None] * (float(positions[n + i]) - positions[at].astype(np.float64))
        top = x.max(axis=1, keepdims=True)
        e = np.exp(x - top)
        lse[i] = top[:, 0] + np.log(e.sum(axis=1))
        e /= e.sum(axis=1, keepdims=True)
        p[i][:, at] = e
        out[i] = e @ v[at]
    return out, lse, p


def commit_slots(n, n_new, count=None, path=None):
    """Slots that the tokens behind the n old ones come from, in order."""
    count = n_new if count is None else count
    return [n + (i if path is None else int(path[i])) for i in range(count)]


def evict_moves(weights, positions, n, budget, recent):
    """(from, to) of every token that moves: kept ones beyond the budget into the free slots below it, both ascending."""
    if n <= budget:
        return []
    newest = int(positions[:n].max())

    def rank(j):
        w = float(weights[j])
        if int(positions[j]) > newest - recent:
            return 0, 0.0, j
        return (1, 0.0, j) if np.isnan(w) else (2, -w, j)

    kept = set(sorted(range(n), key=rank)[:budget])
    free = [j for j in range(budget) if j not in kept]
    return list(zip(sorted(j for j in kept if j >= budget), free))
