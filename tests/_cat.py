"""Plain 64-bit forms of the categorical-head calls, on the CPU with NumPy: rows are sorted, filtered and summed one by one.
Also the bytes of an 8-bit matrix."""
import numpy as np

FMAX = np.float32(np.finfo(np.float32).max)


def scaled(logits32, temperature):
    """Scaled logits (float32 values): -inf where masked, finite elsewhere; and 1 / temperature."""
    T = np.float32(temperature)
    inv = np.float32(1.0) / T if T > 0 else np.float32(1.0)
    with np.errstate(all="ignore"):
        t = np.clip((logits32 * inv).astype(np.float32), -FMAX, FMAX)
    return np.where(np.isnan(logits32) | (logits32 == -np.inf), np.float32(-np.inf), t).astype(np.float32), inv


def kept(logits32, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens kept, most likely first; their log probabilities; summary row) of one row."""
    t, inv = scaled(logits32, temperature)
    live = np.flatnonzero(t > -np.inf)
    if live.size == 0:
        return live, np.zeros(0), np.array([-np.inf, np.inf, -1, 0, inv], np.float64)
    order = live[np.lexsort((live, -t[live].astype(np.float64)))]
    if not temperature > 0:
        top_k, top_p = 1, 1.0
    if 0 < top_k < order.size:
        order = order[:top_k]
    m = np.float64(t[order[0]])
    w = np.exp(t[order].astype(np.float64) - m)
    n = order.size
    if top_p < 1:
        c = np.cumsum(w)
        n = max(1, int(np.sum(np.concatenate([[0.0], c[:-1]]) < np.float64(np.float32(top_p)) * c[-1])))
    if min_p > 0:
        n = min(n, max(1, int(np.sum(w >= min(np.float64(np.float32(min_p)), 1.0)))))
    order, w = order[:n], w[:n]
    norm = m + np.log(w.sum())
    return order, t[order].astype(np.float64) - norm, np.array([norm, t[order[-1]], order[-1], n, inv], np.float64)


def probabilities(logits32, **f):
    order, logp, row = kept(logits32, **f)
    p = np.zeros(logits32.size)
    p[order] = np.exp(logp)
    return p, row


def pick(weights, u):
    """First index whose cumulative weight reaches u times the sum, and how near u is to the border it fell beside."""
    c = np.cumsum(weights.astype(np.longdouble))
    if not c[-1] > 0:
        return -1, 1.0
    at = int(np.searchsorted(c, np.longdouble(u) * c[-1], side="left"))
    return min(at, weights.size - 1), float(np.min(np.abs(c / c[-1] - np.longdouble(u))))


def e4m3(byte):
    byte = np.asarray(byte, np.uint8).astype(np.int64)
    s, e, m = np.where(byte >> 7, -1.0, 1.0), (byte >> 3) & 15, byte & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    return np.where((e == 15) & (m == 7), np.nan, s * v)


def dequantize(data, scale):
    """float64 values of an 8-bit matrix (all padded columns)."""
    rows, ld = data.shape
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))[:, : ld // 128]
    return (e4m3(data).reshape(rows, -1, 128) * s[:, :, None]).reshape(rows, ld)


def scale_bytes(y):
    """The smallest power of two under which each block of 128 fits 448 (float64 rows of whole blocks)."""
    a = np.abs(y).reshape(y.shape[0], -1, 128).max(2)
    m, e = np.frexp(a)
    b = np.where(m > 0.875, e - 8, e - 9) + 127
    return np.where(a == 0, 127, np.clip(b, 0, 254)).astype(np.uint8)
