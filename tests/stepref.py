"""Plain models of a generation step's operators for the tests (numpy, 64 bits): the
position rotation with its roundings, attention over latents, beam search's choice."""
import numpy as np


def turns(pos, freqs):
    """cos and sin of pos * freqs, from 64 bits rounded to fp32: [n, pairs] each."""
    theta = np.asarray(pos, np.float64)[:, None] * np.asarray(freqs, np.float32).astype(np.float64)
    return np.cos(theta).astype(np.float32), np.sin(theta).astype(np.float32)


def turned(x, pos, freqs, interleaved):
    """Rows x [n, heads, d] (fp32 of 16-bit values) turned, every step in fp32 as defined."""
    x = np.asarray(x, np.float32)
    c, s = (t[:, None] for t in turns(pos, freqs))
    r, y = len(freqs), x.copy()
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if interleaved else (slice(0, r), slice(r, 2 * r))
    with np.errstate(all="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def frequencies(dim, base=10000.0):
    return (base ** (-np.arange(0, dim, 2) / dim)).astype(np.float32)


def attend(q, qr, c, r, scale):
    """One row of one head over tokens c [n, latent], r [n, rope]: out, lse, p."""
    if len(c) == 0:
        return np.zeros(c.shape[1]), -np.inf, np.zeros(0)
    x = (c @ q + r @ qr) * scale
    m = x.max()
    e = np.exp(x - m)
    p = e / e.sum()
    return p @ c, m + np.log(e.sum()), p


def choose(logits, scores, k, ended=None, pad=0):
    """A group's candidates: logits [W, V], scores [W]: (t, beam, token) [k] each; the beam within the group."""
    W, V = logits.shape
    x, a = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    found = []
    for b in range(W):
        if np.isnan(a[b]) or a[b] == np.inf:
            return np.full(k, np.nan), np.full(k, -1), np.full(k, -1)
        if ended is not None and ended[b]:
            if a[b] > -np.inf:
                found.append((-a[b], b, pad))
            continue
        if a[b] == -np.inf:
            continue
        m = x[b].max()
        if np.isnan(x[b]).any() or m == np.inf:
            return np.full(k, np.nan), np.full(k, -1), np.full(k, -1)
        if m == -np.inf:
            continue
        t = a[b] + (x[b] - (m + np.log(np.exp(x[b] - m).sum())))
        best = np.lexsort((np.arange(V), -x[b]))[:k]             # within a row t follows x
        found += [(-t[v], b, v) for v in best if x[b][v] > -np.inf]
    found.sort()
    found = found[:k] + [(np.inf, -1, -1)] * max(0, k - len(found))
    t, b, v = zip(*found)
    return -np.array(t), np.array(b), np.array(v)
