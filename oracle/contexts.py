"""Plain float64 definitions of the operators for long and shared contexts (numpy only), with bounds on the rounding
error that a bf16-in, fp32-accumulating implementation may make.

Arrays are float64; K, V are [n, hd] for one (sequence, head).  Every attention returns (out, tol): |computed - out| <= tol
holds for an implementation that
  * computes scores and sums in fp32, a step 2^-23 lost per operation (tensor-core adds may truncate),
  * takes 2^x with an error of 2^-22 relative,
  * rounds the softmax weights to bf16 where they meet V (``p_bf16``: 2^-8 relative) or not,
  * rounds the result to bf16 (2^-8 relative).
A score error of e (log2 units) moves a weight by a factor within 2^(+-e), in numerator and denominator.
"""
import numpy as np

STEP, BF16 = 2.0 ** -23, 2.0 ** -8
LOG2E = 1.4426950408889634


def attend(q, K, V, scale=None, p_bf16=False):
    """One query [hd] over rows K, V [n, hd]: (out [hd], weights [n], tol on out [hd], relative tol on the weights)."""
    hd = q.shape[0]
    n = K.shape[0]
    if n == 0:
        return np.zeros(hd), np.zeros(0), np.zeros(hd), 0.0
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    s = K @ q * scale
    e = np.exp(s - s.max())
    p = e / e.sum()
    out = p @ V
    score_err = (np.abs(K) @ np.abs(q)).max() * scale * LOG2E * (hd + 4) * STEP
    rel = 2 * np.log(2.0) * score_err + (n + 16) * STEP + 4 * 2.0 ** -22
    mass = p @ np.abs(V)
    tol = (rel + (BF16 if p_bf16 else 0.0)) * mass
    return out, p, tol + BF16 * (np.abs(out) + tol) + 1e-30, rel


def window_rows(n, window, sinks):
    """Rows that the query of row n - 1 sees."""
    return [j for j in range(n) if j < sinks or j >= n - window]


def decode_window(q, K, V, n, window, sinks):
    """q [B,H,hd], K, V [B,H,N,hd], n [B]: (out, tol)."""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(q.shape[0]):
        rows = window_rows(int(n[b]), window, sinks)
        for h in range(q.shape[1]):
            out[b, h], _, tol[b, h], _ = attend(q[b, h], K[b, h, rows], V[b, h, rows])
    return out, tol


def prefill_window(q, K, V, window, sinks, positions=None):
    """q [T,hd], K, V [T,hd] of one (sequence, head): (out, tol) at the given positions."""
    positions = range(q.shape[0]) if positions is None else positions
    got = []
    for t in positions:
        rows = window_rows(t + 1, window, sinks)
        o, _, e, _ = attend(q[t], K[rows], V[rows], p_bf16=True)
        got.append((o, e))
    return np.array([g[0] for g in got]), np.array([g[1] for g in got])


def decode_shared(q, PK, PV, S, K, V, n):
    """q [B,H,hd]; prefix PK, PV [H,cap,hd] of S rows; own K, V [B,H,N,hd] of n[b] rows: (out, tol)."""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            k = np.concatenate([PK[h, :S], K[b, h, :n[b]]])
            v = np.concatenate([PV[h, :S], V[b, h, :n[b]]])
            out[b, h], _, tol[b, h], _ = attend(q[b, h], k, v, p_bf16=True)
    return out, tol


def decode_weights(q, K, V, n, sums, fresh=None):
    """(out, tol, new sums, tol on them); fresh[b]: a row whose sum starts now, or -1."""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    new, new_tol = sums.astype(np.float64).copy(), np.zeros(sums.shape)
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            m = int(n[b])
            out[b, h], p, tol[b, h], rel = attend(q[b, h], K[b, h, :m], V[b, h, :m])
            old = new[b, h, :m].copy()
            if fresh is not None and fresh[b] >= 0:
                old[fresh[b]] = 0.0
            new[b, h, :m] = old + p
            new_tol[b, h, :m] = rel * p + STEP * np.abs(new[b, h, :m]) + 1e-30
    return out, tol, new, new_tol


def evicted(sums, n, n_keep, n_sinks, n_recent):
    """Rows of one (sequence, head) of n rows that stay, in order (n > n_keep)."""
    middle = list(range(n_sinks, n - n_recent))
    value = lambda j: -np.inf if np.isnan(sums[j]) else float(sums[j])   # noqa: E731
    # a NaN is below every number, minus infinity included; ties go to the lowest index
    middle.sort(key=lambda j: (-value(j), bool(np.isnan(sums[j])), j))
    best = middle[:n_keep - n_sinks - n_recent]
    return sorted(list(range(n_sinks)) + best + list(range(n - n_recent, n)))
