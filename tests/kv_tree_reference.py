"""Trees over a paged cache, verification, weights, choice and move from their definitions, in 64 bits on the host, sequence by sequence."""
import math

import numpy as np


def ancestors(parents):
    """Rows that each row of a tree sees [rows, rows]: those on the way to it, and itself."""
    n = len(parents)
    seen = np.eye(n, dtype=bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            seen[i] |= seen[p]
    return seen


def words(seen, stride, junk=None):
    """Masks as int64 [rows, stride]; `junk`: bits behind the last row."""
    n = seen.shape[0]
    bits = np.zeros((n, stride * 64), dtype=np.uint64)
    bits[:, :seen.shape[1]] = seen
    if junk is not None:
        bits[:, seen.shape[1]:] = junk
    return (bits.reshape(n, stride, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)


def visible(seen, tokens, window=0):
    """Which tokens each row of a tree sees [rows, tokens]."""
    n = seen.shape[0]
    base = tokens - n
    out = np.zeros((n, tokens), dtype=bool)
    for r in range(n):
        lo = max(0, base + int(seen[r].sum()) - window) if window else 0
        out[r, lo:max(base, 0)] = True
        for j in np.flatnonzero(seen[r]):
            if base + j >= 0:
                out[r, base + j] = True
    return out


def spans(rows, tokens, window=0, causal=True):
    """Which tokens each of the last rows of a sequence sees [rows, tokens]."""
    t = np.arange(tokens)
    hi = (tokens - rows + np.arange(rows) + 1 if causal else np.full(rows, tokens))[:, None]
    return (t < hi) & ((t >= hi - window) if window else True)


def attend(q, k, v, seen, scale):
    """One sequence, any mask [rows, tokens]: as kv_reference.attend."""
    rows, q_heads, dim = q.shape
    group = q_heads // k.shape[1]
    out, lse = np.zeros((rows, q_heads, dim)), np.full((rows, q_heads), -math.inf)
    mass, size = np.zeros((rows, q_heads, dim)), np.zeros((rows, q_heads))
    for r in range(rows):
        at = np.flatnonzero(seen[r])
        if not len(at):
            continue
        for h in range(q_heads):
            kk, vv = k[at, h // group], v[at, h // group]
            s = kk @ q[r, h] * scale
            top = s.max()
            w = np.exp(s - top)
            lse[r, h] = top + math.log(w.sum())
            w = w / w.sum()
            out[r, h] = w @ vv
            mass[r, h] = w @ np.abs(vv)
            size[r, h] = scale * (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, lse, mass, size


def weigh(q, k, lse, seen, scale):
    """One sequence: weights [heads, tokens], and what bounds their error in 32 bits.  A score's sum of `dim` products is off by
    (dim + 8) 2^-24 of its absolute terms; the exponent by 2^-24 of what it is made of, scaled by log2(e), four roundings at most; the
    exponential by 2^-23; and each sum by 2^-24 a term.  An exponential below the least normal number may be 0."""
    rows, q_heads, dim = q.shape
    heads, e = k.shape[1], 2.0 ** -24
    group = q_heads // heads
    out, off = np.zeros((heads, k.shape[0])), np.zeros((heads, k.shape[0]))
    for r in range(rows):
        at = np.flatnonzero(seen[r])
        for h in range(q_heads):
            if not math.isfinite(lse[r, h]) or not len(at):
                continue
            kk = k[at, h // group]
            s = kk @ q[r, h] * scale
            w = np.exp(s - lse[r, h])
            size = scale * (np.abs(kk) @ np.abs(q[r, h]))
            out[h // group, at] += w
            off[h // group, at] += w * ((dim + 8) * e * size + 4 * e * (np.abs(s) + abs(lse[r, h])) + 2 * e) + 2.0 ** -126
    return out, off + (rows * group + 64) * e * out


def sound(p):
    p = p.astype(np.float64)
    return np.where((p > 0) & (p < math.inf), p, 0.0)


def verify(target, draft, tokens, parents, accept, next_):
    """One sequence: target and draft [rows, vocab] in 64 bits -> path, token."""
    n, vocab = target.shape
    at, path = 0, [0]
    r, mass, gone = sound(target[0]), 1.0, set()
    for i in range(1, n):
        if parents[i] != at:
            continue
        x, inside = int(tokens[i]), 0 <= tokens[i] < vocab
        rx = r[x] if inside else 0.0
        if draft is not None:
            q = sound(draft[at])
            stands = accept[i] * (q[x] if inside else 0.0) < rx
        else:
            stands = accept[i] * mass < rx
        if stands:
            at = i
            path.append(i)
            r, mass = sound(target[i]), 1.0
        elif draft is not None:
            r = np.maximum(r - q, 0.0)
            r = r / r.sum() if r.sum() > 0 else r
        else:
            mass = max(mass - rx, 0.0)
            if inside:
                r = r.copy()
                r[x] = 0.0
    if not r.sum() > 0:
        r = sound(target[at])
    if not r.sum() > 0:
        return path, -1
    total = np.cumsum(r)
    over = np.flatnonzero(total > next_ * total[-1])
    return path, int(over[0]) if len(over) else int(np.flatnonzero(r)[-1])


def choose(weights, budget, first, recent):
    """One list of the weights of all tokens of a sequence -> the tokens that stay."""
    n = len(weights)
    if n <= budget:
        return list(range(n))
    w = np.where(np.isnan(weights), -math.inf, weights)
    always = set(range(first)) | set(range(n - recent, n))
    others = [t for t in np.lexsort((np.arange(n), -w)) if int(t) not in always]
    return sorted(list(always) + [int(t) for t in others[:budget - len(always)]])
