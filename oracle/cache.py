"""The cache operators in plain fp64 NumPy, from their definitions: which tokens a draft's
queries attend to, their attention, the weights that cached tokens receive, eviction by
those weights and the compaction of the cache.  One (batch row, KV head) at a time."""

import math

import numpy as np

from . import method as M


def visible(T, n, N, L, w, sel=None, bits=None):
    """[N, T + n] flags: the tokens that each of N queries attends to.  T context tokens; sel None: all of them, else
    the union of the selected blocks and the last w; bits: mask words of n drafted tokens, None without a draft."""
    see = np.zeros((N, T + n), dtype=bool)
    context = range(T) if sel is None else M.union_tokens(T, L, w, sel)
    see[:, list(context)] = True
    if bits is not None:
        for i in range(N):
            for j in range(n):
                see[i, T + j] = bool((int(bits[i]) >> j) & 1)
        see[n:] = False
    return see


def _scores(q, K, see, c):
    """c q.k [N, G, tokens], -inf where a query does not attend (whatever the key holds)."""
    N, G, d = q.shape
    t = np.nonzero(see.any(0))[0]
    s = np.full((N, G, see.shape[1]), -np.inf)
    s[:, :, t] = c * (q.reshape(N * G, d) @ K[t].T).reshape(N, G, len(t))
    return np.where(see[:, None, :], s, -np.inf)


def tree_attention(q, K, V, see, c):
    """q [N, G, d], K and V [tokens, d], see [N, tokens]: out [N, G, d] and lse [N, G]; 0 and -inf for a query that
    attends to nothing.  A value enters only the queries that attend to its token."""
    N, G, d = q.shape
    s = _scores(q, K, see, c)
    out, lse = np.zeros((N, G, d)), np.full((N, G), -np.inf)
    for i in range(N):
        t = np.nonzero(see[i])[0]
        if len(t) == 0:
            continue
        top = s[i][:, t].max(1, keepdims=True)
        p = np.exp(s[i][:, t] - top)
        total = p.sum(1, keepdims=True)
        out[i] = (p @ V[t]) / total
        lse[i] = (top + np.log(total))[:, 0]
    return out, lse


def attention_weights(q, K, see, lse, c):
    """Sum over queries and heads of exp(c q.k - lse) per token [tokens]; a head whose lse is infinite adds nothing."""
    s = _scores(q, K, see, c)
    adds = see[:, None, :] & ~np.isinf(lse)[:, :, None]      # (inf - inf of a key's infinity is no term either)
    return np.exp(np.where(adds, s - np.where(np.isinf(lse), 0.0, lse)[:, :, None], -np.inf)).sum((0, 1))


def evict(weights, T, keep, sinks, recent):
    """Kept positions, ascending, of T tokens."""
    if T <= keep:
        return list(range(T))
    w = [-math.inf if math.isnan(x) else x for x in np.asarray(weights, dtype=np.float64)[:T].tolist()]
    middle = sorted(range(sinks, T - recent), key=lambda t: (-w[t], t))[:keep - sinks - recent]
    return sorted(list(range(sinks)) + middle + list(range(T - recent, T)))


def compact(rows, out, kept, T, first):
    """out with out[first + j] = rows[kept[j]] for the entries in [0, T) that fit."""
    src = np.array(rows, copy=True)
    for j, t in enumerate(kept):
        if 0 <= t < T and first + j < len(out):
            out[first + j] = src[t]
    return out


def compact_weights(weights, out, kept, T, first):
    """The same for weights, with 0 for entries that move nothing and behind the last entry up to T."""
    src = np.array(weights, copy=True)
    for j in range(max(len(kept), T - first)):
        if first + j < len(out):
            t = kept[j] if j < len(kept) else -1
            out[first + j] = src[t] if 0 <= t < T else 0.0
    return out
