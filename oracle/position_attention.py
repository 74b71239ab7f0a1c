"""CPU ORACLE -- TEST INFRASTRUCTURE ONLY (never imported by the product path).

Attention over one token sequence (a document), and rotary positions, in fp64 numpy with full score rows:

    x[h,i,j] = (q[i,h] . k[j,h']) / sqrt(d),  h' = h / (H / G)       S = cap tanh(x / cap) (cap 0: x) - slopes[h] |i - j|
    query i sees key j  iff  not causal, or j <= i, or j < prefix
    P = softmax_j S,  O = P V,  LSE = log sum_j exp S

Backward for L = sum(O dO) by the chain rule: dP = dO V^T, dS = P (dP - sum_j P dP), dX = dS (1 - tanh^2), dq = dX k / sqrt(d),
dk = sum over the heads of a key head of dX^T q / sqrt(d), dv likewise of P^T dO.  A packed batch is a loop over documents.

Beside the values, `bounds` gives how far a result may be off when the probabilities, the score gradients and the results are rounded to
bf16, half a step (2^-8) each, and everything else is fp32; `norms` the 2-norm of a whole result's error when those roundings are
independent of one another, where a rounding is off by at most 2^-8 / sqrt(3) in the mean square.  (A limit relative to the result's own
norm would not do: the sum of a row's score gradients is 0, so a part that all keys have in common cancels in dq, but not in the error.)
"""
from __future__ import annotations

import numpy as np

def _rows_times(a, x):
    """sum_j a[h,i,j] x[j,h,d]."""
    return np.matmul(a, x.transpose(1, 0, 2)).transpose(1, 0, 2)


def _columns_times(a, x):
    """sum_i a[h,i,j] x[i,h,d]."""
    return np.matmul(a.transpose(0, 2, 1), x.transpose(1, 0, 2)).transpose(1, 0, 2)


def _products(x, y):
    """sum_c x[i,h,c] y[j,h,c]."""
    return np.matmul(x.transpose(1, 0, 2), y.transpose(1, 2, 0))


def _weighed(a, x):
    """sum_ij a[h,i,j] sum_d x[i,h,d]."""
    return (a.sum(2) * x.sum(2).T).sum()


HALF_STEP = 2.0 ** -8          # bf16
MEAN_STEP = HALF_STEP / 3 ** 0.5


def scores(q, k, causal, prefix, slopes, cap):
    """S [H, n, n] with -inf where masked, tanh(x / cap) (zeros without a cap), and sum_c |q_c k_c| / sqrt(d)."""
    n, H, d = q.shape
    kk = np.repeat(k, H // k.shape[1], axis=1)
    with np.errstate(invalid="ignore"):
        x = _products(q, kk) / np.sqrt(d)
        size = _products(np.abs(q), np.abs(kk)) / np.sqrt(d)
    t = np.tanh(x / cap) if cap else np.zeros_like(x)
    s = cap * t if cap else x
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    if slopes is not None:
        s = s - slopes[:, None, None] * np.abs(i - j)
    if causal:
        s = np.where((j <= i) | (j < prefix), s, -np.inf)
    return s, t, size


def attention(q, k, v, dout=None, causal=False, prefix=0, slopes=None, cap=0.0):
    """q, dout fp64 [n,H,d]; k, v [n,G,d]; slopes [H].  Returns a dict: out [n,H,d], lse [H,n], with dout dq, dk, dv, and `bounds`, the
    same keys: elementwise limits of the error (dq and dk: with the forward's fp32 output; `dq_own`, `dk_own` where the backward sums Delta itself,
    from probabilities in fp32; `dq_out`, `dk_out` if it were made of the bf16 output), and `norms`."""
    n, H, d = q.shape
    G = k.shape[1]
    vv, kk = np.repeat(v, H // G, axis=1), np.repeat(k, H // G, axis=1)
    s, t, size = scores(q, k, causal, prefix, slopes, cap)
    top = s.max(2, keepdims=True)
    e = np.exp(s - top)
    l = e.sum(2, keepdims=True)
    p = e / l
    out = _rows_times(p, vv)
    lse = (top + np.log(l))[:, :, 0]
    # fp32: products summed in the tensor core (d terms and one for the fold of lse), the tanh's polynomial, exponent and penalty
    slip = 2.0 ** -22 * (d * size + np.abs(lse)[:, :, None]) + 1e-6 * size + 2e-6 + 2.0 ** -21 * np.where(np.isfinite(s), np.abs(s), 0.0)
    drift = (p * slip).sum(2) + 1e-6                       # of a row's log-sum-exp
    wrong = slip + drift[:, :, None]                       # relative, of a probability
    near = _rows_times(p * (HALF_STEP + wrong), np.abs(vv)) * 1.01
    out32 = near + (HALF_STEP + drift.T[:, :, None]) * np.abs(out)          # (the normaliser is rounded, too, or not)
    r = {"out": out, "lse": lse, "bounds": {"out": out32 + HALF_STEP * np.abs(out) * 1.01, "lse": drift}}
    squares = lambda x: (x * x).sum()  # noqa: E731
    # (the values as they are: their mean over a row is taken off where the normaliser is rounded alike, which can only make it less)
    r["norms"] = {"out": MEAN_STEP * np.sqrt(_weighed((p * p).transpose(0, 2, 1), vv * vv) + squares(out))}
    if dout is None:
        return r
    dp = _products(dout, vv)
    delta = (p * dp).sum(2, keepdims=True)
    g = 1.0 - t * t
    dx = p * (dp - delta) * g

    def heads(x):
        return x.reshape(n, G, H // G, d).sum(2)

    r["dq"] = _rows_times(dx, kk) / np.sqrt(d)
    r["dk"] = heads(_columns_times(dx, q)) / np.sqrt(d)
    r["dv"] = heads(_columns_times(p, dout))
    b = r["bounds"]
    sized = _products(np.abs(dout), np.abs(vv))
    tail = 2.0 ** -22 * d * (sized + (np.abs(dout) * np.abs(out)).sum(2).T[:, :, None])
    for key, off in (("", out32), ("_out", b["out"])):
        off_delta = (np.abs(dout) * off).sum(2).T[:, :, None]
        off_x = 1.01 * ((HALF_STEP + wrong) * np.abs(dx) + p * (g + 4e-6) * (off_delta + tail) + p * np.abs(dp - delta) * 4e-6)
        b["dq" + key] = _rows_times(off_x, np.abs(kk)) / np.sqrt(d) + HALF_STEP * 1.01 * np.abs(r["dq"]) + 1e-30
        b["dk" + key] = heads(_columns_times(off_x, np.abs(q))) / np.sqrt(d) + HALF_STEP * 1.01 * np.abs(r["dk"]) + 1e-30
    # Delta of the backward's own probabilities, in fp32: what they are off, less what they have in common, and the sums
    off_delta = (p * wrong * np.abs(dp - delta)).sum(2, keepdims=True) + (p * tail).sum(2, keepdims=True)
    off_x = 1.01 * ((HALF_STEP + wrong) * np.abs(dx) + p * (g + 4e-6) * (off_delta + tail) + p * np.abs(dp - delta) * 4e-6)
    b["dq_own"] = _rows_times(off_x, np.abs(kk)) / np.sqrt(d) + HALF_STEP * 1.01 * np.abs(r["dq"]) + 1e-30
    b["dk_own"] = heads(_columns_times(off_x, np.abs(q))) / np.sqrt(d) + HALF_STEP * 1.01 * np.abs(r["dk"]) + 1e-30
    r["norms"]["dq_own"] = MEAN_STEP * np.sqrt(_weighed((dx * dx).transpose(0, 2, 1), kk * kk) / d + squares(r["dq"]))
    r["norms"]["dk_own"] = MEAN_STEP * np.sqrt(_weighed(dx * dx, q * q) / d + squares(r["dk"]))
    # Delta with the fp32 output: sum_j of (a probability's rounding) P (dP - Delta), since the rounded normaliser takes the mean off
    off_delta2 = ((p * (dp - delta)) ** 2).sum(2)
    pull = _rows_times(p * g, kk)
    r["norms"]["dq"] = MEAN_STEP * np.sqrt((_weighed((dx * dx).transpose(0, 2, 1), kk * kk) + (off_delta2.T[:, :, None] * pull * pull).sum()) / d + squares(r["dq"]))
    r["norms"]["dk"] = MEAN_STEP * np.sqrt(_weighed(dx * dx + (p * g) ** 2 * off_delta2[:, :, None], q * q) / d + squares(r["dk"]))
    r["norms"]["dv"] = MEAN_STEP * np.sqrt(_weighed(p * p, dout * dout) + squares(r["dv"]))
    b["dv"] = heads(_columns_times(1.01 * p * (HALF_STEP + wrong), np.abs(dout))) + HALF_STEP * 1.01 * np.abs(r["dv"]) + 1e-30
    return r


def batch_attention(q, k, v, dout, cu, causal=False, prefix=None, slopes=None, cap=0.0):
    """The same for a packed batch: rows cu[g] .. cu[g+1]-1 are document g; NaN in the rows of no document."""
    T, H, _ = q.shape
    r = {"out": np.full(q.shape, np.nan), "lse": np.full((H, T), np.nan), "bounds": {}, "norms": {}}
    if dout is not None:
        r |= {"dq": np.full(q.shape, np.nan), "dk": np.full(k.shape, np.nan), "dv": np.full(k.shape, np.nan)}
    for g in range(len(cu) - 1):
        a, b = int(cu[g]), int(cu[g + 1])
        if a == b:
            continue
        one = attention(q[a:b], k[a:b], v[a:b], None if dout is None else dout[a:b], causal, 0 if prefix is None else int(prefix[g]), slopes, cap)
        for key, x in one["norms"].items():
            r["norms"][key] = float(np.hypot(r["norms"].get(key, 0.0), x))
        for key, into in [(x, r) for x in one if x not in ("bounds", "norms")] + [(x, r["bounds"]) for x in one["bounds"]]:
            x = one["bounds"][key] if into is r["bounds"] else one[key]
            if into is r["bounds"] and key not in into:
                into[key] = np.full((H, T) if key == "lse" else (T,) + x.shape[1:], np.nan)
            if key == "lse":
                into[key][:, a:b] = x
            else:
                into[key][a:b] = x
    return r


def rotate(x, frequencies, positions, interleaved, scale=1.0, inverse=False):
    """Rotary positions of x fp64 [T, heads, d]: the first 2 len(frequencies) channels of every head."""
    half = len(frequencies)
    w = np.asarray(positions, np.longdouble)[:, None] * np.asarray(frequencies, np.longdouble)[None, :]
    c, s = (scale * np.cos(w)).astype(np.float64)[:, None], ((-scale if inverse else scale) * np.sin(w)).astype(np.float64)[:, None]
    y = np.array(x, np.float64)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y
