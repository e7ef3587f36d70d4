"""float64 position operators of attention (test infrastructure).

The paper's stages use neither; both are options of this library's attention.

* Norms and rotation of the query and key heads: per token and head,
  n = x / sqrt(mean(x^2) + eps) * gain, then the first R elements of n in pairs
  (i, i + R/2) ("half") or (2i, 2i + 1) ("adjacent"), pair i turned by the angle
  position * freq[i].
* Relative position bias: the score of query i and key j adds
  table[bucket(i - j), head], where bucket(n) counts the bounds[1:] at or below
  min(n, max_distance); entries at or below -2^15 hide their distances, larger ones than
  2^15 count as it.
"""
import numpy as np


def freqs(theta, R):
    """theta^(-2 i / R), i < R / 2."""
    return np.array([theta ** (-2.0 * i / R) for i in range(R // 2)], np.float64)


def _pair_index(R, pairs):
    i = np.arange(R // 2)
    return (i, i + R // 2) if pairs == "half" else (2 * i, 2 * i + 1)


def rotate(x, pos, freq, pairs, sign=1):
    """Heads x [T, H, dh] with the first 2 len(freq) elements turned by sign * pos * freq."""
    R = 2 * len(freq)
    a, b = _pair_index(R, pairs)
    ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(freq, np.float64)
    c, s = np.cos(ang), sign * np.sin(ang)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def norm_rope_fwd(x, gain, pos, freq, pairs="half", eps=1e-5):
    """x [T, H, dh]; gain [H, dh] or None (no norm); freq empty: no rotation."""
    n = x if gain is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    return rotate(n, pos, freq, pairs) if len(freq) else n.copy()


def norm_rope_bwd(dy, x, gain, pos, freq, pairs="half", eps=1e-5):
    """Returns (dx, dgain [H, dh] or None): the rotation back, then the norm's backward."""
    dn = rotate(dy, pos, freq, pairs, -1) if len(freq) else dy
    if gain is None:
        return dn, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh = x * r
    e = dn * gain
    return r * (e - xh * (e * xh).mean(-1, keepdims=True)), (dn * xh).sum(0)


def bounds(n_buckets, max_distance):
    """First distance of every bucket: n for n < e = n_buckets // 2, then the first whole
    distance d with (d / e)^m >= (max_distance / e)^k, m = n_buckets - e, in whole numbers."""
    e = n_buckets // 2
    m, out, d = n_buckets - e, list(range(e + 1)), e
    for k in range(1, m):
        while d ** m < e ** (m - k) * max_distance ** k:
            d += 1
        out.append(d)
    return out[:n_buckets]


def buckets(bnd, max_distance, S):
    """Bucket of every distance 0 .. S - 1."""
    return np.array([sum(b <= min(n, max_distance) for b in bnd[1:]) for n in range(S)])


def bias_by_distance(table, bnd, max_distance, S):
    """[H, S] bias of each head at every distance (hidden ones -inf)."""
    t = np.minimum(np.asarray(table, np.float64), 2.0 ** 15)
    t[t <= -2.0 ** 15] = -np.inf
    return t[buckets(bnd, max_distance, S)].T


def table_grad(ds, bnd, max_distance):
    """ds [H, S, S] (summed over sequences) -> [n_buckets, H]: sums over the pairs of each bucket."""
    H, S, _ = ds.shape
    g = np.zeros((len(bnd), H))
    b = buckets(bnd, max_distance, S)
    for n in range(S):
        g[b[n]] += np.trace(ds, offset=-n, axis1=1, axis2=2)
    return g
