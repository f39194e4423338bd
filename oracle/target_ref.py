"""CPU oracle of the target's operators between its linears: norms and rotation with
the cache append, causal attention over the cache, verification of drafted tokens.

TEST INFRASTRUCTURE ONLY.  Only ``tests/`` may import it.  It shares no code with
``paper_2607_04244_amd`` and imports nothing from it.

Definitions (Kim, Lee, Kim, arXiv 2607.04244, Sec. 2.2: the target verifies a draft
block in one forward pass, and the loop keeps a prefix, without loss):

* A sequence of L cached tokens whose last n are new: new token i is at position
  L - n + i, and sees the keys j <= its position.
* norm: x / sqrt(mean(x^2) + eps) * w over the 128 dimensions of a head; rotation by
  position * inv_freq of the pairs (i, i + R/2) or (2i, 2i + 1).
* Verification: drafted token x_i stays while u_i Q_i(x_i) < P_i(x_i); at the first
  that does not the next token is drawn from max(P - Q, 0), and from P behind the last
  drafted token, by the running sum in index order.

Plain numpy, float64.  Pinned by ``tests/test_oracle_target.py``.
"""

import math

import numpy as np

HEAD = 128


def bf16_to_f64(bits):
    """bf16 bit patterns (uint16) -> float64 values, exactly."""
    u = np.asarray(bits, dtype=np.uint16).astype(np.uint32) << np.uint32(16)
    return u.view(np.float32).astype(np.float64)


def norm(x, w, eps):
    """x [..., 128] float64, w [128] float64 or None."""
    if w is None:
        return x
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * w


def rotate(x, position, inv_freq, interleaved):
    """x [heads, 128] of the token at an (integer) position."""
    y = x.copy()
    half = len(inv_freq)
    for i in range(half):
        a = position * float(inv_freq[i])
        i0, i1 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[:, i0] = x[:, i0] * math.cos(a) - x[:, i1] * math.sin(a)
        y[:, i1] = x[:, i0] * math.sin(a) + x[:, i1] * math.cos(a)
    return y


def positions(new, length):
    """[(sequence, position)] of every new token in row order."""
    return [(b, L - n + i) for b, (n, L) in enumerate(zip(new, length)) for i in range(n)]


def causal_attention(q, keys, values, scale):
    """One sequence: q [n, Hq, 128] its new tokens, keys and values [L, Hkv, 128],
    all float64.  Returns (out, spread) [n, Hq, 128] with spread = sum_j p_j |v_j|."""
    n, Hq, _ = q.shape
    L, Hkv, _ = keys.shape
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(n):
        seen = L - n + i + 1
        if seen <= 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = keys[:seen, g] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ values[:seen, g]
            spread[i, h] = p @ np.abs(values[:seen, g])
    return out, spread


def _distribution(logits, T):
    """Probabilities of a row of float64 logits; -inf and NaN are masked."""
    x = np.where(np.isnan(logits), -np.inf, logits)
    m = x.max()
    p = np.zeros(len(x))
    if m == -np.inf:
        return p
    if not T > 0:
        p[int(np.argmax(x == m))] = 1.0
        return p
    on = x > -np.inf
    below = x[on] - m if np.isfinite(m) else np.full(on.sum(), -np.inf)
    p[on] = np.exp(np.where(x[on] == m, 0.0, below) / T)
    return p / p.sum()


def verify(target, draft, drafted, u, T):
    """One sequence: target [n + 1, V] and draft [n, V] (or None) logits, drafted [n],
    u [n] + [the number that draws the next token].  Returns (accepted, next)."""
    n = len(drafted)
    V = target.shape[1]
    w = None
    a = 0
    while a < n:
        p = _distribution(target[a], T)
        x = int(drafted[a])
        inside = 0 <= x < V
        if draft is not None and T > 0:
            q = _distribution(draft[a], T)
            qx = q[x] if inside else 0.0
        else:
            q = np.zeros(V)
            if inside:
                q[x] = 1.0
            qx = 1.0
        if not u[a] * qx < (p[x] if inside else 0.0):
            w = np.maximum(p - q, 0.0)
            if not w.sum() > 0:
                w = p
            break
        a += 1
    if w is None:
        w = _distribution(target[a], T)
    if not w.sum() > 0:
        return a, -1
    c = np.cumsum(w)
    over = np.nonzero(c > u[n] * c[-1])[0]
    return a, int(over[0]) if len(over) else int(np.nonzero(w > 0)[0][-1])
