"""Verification of drafted tokens, sequence by sequence in numpy and 64 bits, from the definitions in cat.h."""
import numpy as np

LARGEST = float(np.finfo(np.float32).max)
LEAST = -1000 * np.log(2)        # an entry of less than 2^-1000 of its row's largest weight has none


def masses(logits, T):
    x = np.asarray(logits, dtype=np.float64)
    x = np.minimum(np.where(np.isnan(x), -np.inf, x), LARGEST)
    top = x.max()
    if top == -np.inf:
        return np.zeros_like(x)
    if not T > 0:
        one = np.zeros_like(x)
        one[int(np.argmax(x))] = 1.0
        return one
    with np.errstate(over="ignore"):
        at = (x - top) / float(T)
    e = np.where(at < LEAST, 0.0, np.exp(np.maximum(at, LEAST)))
    return e / e.sum()


def uniform(u):
    return min(max(0.0 if np.isnan(u) else float(u), 0.0), 1 - 2.0 ** -24)


def draw(mass, u):
    """(first index whose cumulated mass exceeds u times the whole, distance of that decision to the nearest other one)."""
    total = mass.sum()
    if not total > 0:
        return -1, np.inf
    u = uniform(u)
    rising = np.cumsum(mass)
    goal = u * total
    i = int(np.argmax(rising > goal)) if (rising > goal).any() else int(np.flatnonzero(mass > 0)[-1])
    return i, min(rising[i] - goal, goal - (rising[i] - mass[i]) if goal > 0 else np.inf)


def verify(target, draft, tokens, u_accept, u_sample, lengths=None, temperature=None):
    """(tokens [B, S + 1], accepted [B], margin [B]): margin is how far, in mass, the closest decision of a sequence was from the other
    outcome -- sums in 64 bits cannot tell apart what is below 1e-12 or so.  Sequences of negative length give -9."""
    target = np.asarray(target)
    B, S1, V = target.shape
    out, kept, margin = np.full((B, S1), -1, np.int32), np.zeros(B, np.int32), np.full(B, np.inf)
    for b in range(B):
        n = S1 - 1 if lengths is None else min(int(lengths[b]), S1 - 1)
        if n < 0:
            out[b], kept[b] = -9, -9
            continue
        T = 1.0 if temperature is None else float(temperature[b])
        j, refused = 0, False
        while True:
            p = masses(target[b, j], T)
            if j == n:
                break
            x = int(tokens[b, j])
            inside = 0 <= x < V
            if draft is None:
                q = np.zeros(V)
                if inside:
                    q[x] = 1.0
            else:
                q = masses(draft[b, j], T)
            # (by logarithms: the masses may be next to the smallest numbers there are, and their product below)
            with np.errstate(divide="ignore"):
                left, right = np.log(uniform(u_accept[b, j])) + np.log(q[x] if inside else 0.0), np.log(p[x] if inside else 0.0)
            if T > 0 and np.isfinite(left) and np.isfinite(right):
                margin[b] = min(margin[b], abs(left - right))
            if not left < right:
                refused = True
                break
            out[b, j] = x
            j += 1
        if refused:
            rest = np.maximum(p - q, 0)
            if rest.sum() >= 2.0 ** -40:
                p = rest
        kept[b] = j
        out[b, j], m = draw(p, u_sample[b])
        margin[b] = min(margin[b], m)
    return out, kept, margin
