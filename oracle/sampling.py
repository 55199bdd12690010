"""Double-precision oracle of drafting and verifying by sampling (host, numpy): the distributions are written out."""
import math

import numpy as np

U_MOST = 1.0 - 2.0 ** -24


def unit(u):
    u = float(u)
    return min(max(u, 0.0), U_MOST) if u == u else 0.0


def distribution(logits, temperature):
    """-> probabilities, or None where the row is no distribution."""
    z = np.asarray(logits, np.float64) / float(np.float32(temperature))
    if np.isnan(z).any() or z.max() == math.inf or z.max() == -math.inf:
        return None
    e = np.exp(z - z.max())
    return e / math.fsum(e)


def first_over(w, u):
    run = np.cumsum(w)
    return min(int(np.sum(run <= unit(u) * run[-1])), int(np.flatnonzero(w > 0)[-1]))


def draw(logits, temperature, draws, uniforms, most=16):
    out = np.full(most, -1, np.int32)
    p = distribution(logits, temperature)
    if p is None:
        return out
    w = p.copy()
    for j in range(draws):
        if not w.sum() > 0:
            break
        out[j] = first_over(w, uniforms[j])
        w[out[j]] = 0
    return out


def verify(parent, tokens, logits, uniforms, temperature, draft_row=None, draft_logits=None, draft_temperature=1.0):
    """One sequence -> (nodes, tokens emitted)."""
    n, vocab = len(parent), logits.shape[1]
    if n == 0:
        return [], []
    nodes, emitted = [0], []
    while True:
        at = nodes[-1]
        p = distribution(logits[at], temperature)
        d = -1 if draft_row is None else int(draft_row[at])
        if draft_row is not None and d >= len(draft_logits):
            d = -1
        children = [c for c in range(at + 1, n) if parent[c] == at]
        q = distribution(draft_logits[d], draft_temperature) if d >= 0 and children else None
        if p is None:
            return nodes, emitted + [0]
        chosen = None
        if not (d >= 0 and children and q is None):
            for c in children:
                x = int(tokens[c])
                if x < 0 or x >= vocab:
                    continue
                u = unit(uniforms[c])
                if q is None:
                    if u < p[x]:
                        chosen = c
                        break
                    rest = p.copy()
                    rest[x] = 0
                    if rest.sum() > 0:
                        p = rest / rest.sum()
                elif q[x] > 0:
                    if u * q[x] < p[x]:
                        chosen = c
                        break
                    rest = np.maximum(p - q, 0)
                    if rest.sum() > 0:
                        p = rest / rest.sum()
                    q[x] = 0
                    if q.sum() > 0:
                        q = q / q.sum()
        if chosen is None:
            return nodes, emitted + [first_over(p, uniforms[0])]
        nodes.append(chosen)
        emitted.append(int(tokens[chosen]))
