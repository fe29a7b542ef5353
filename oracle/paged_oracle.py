"""The paged token cache in plain NumPy: quantised rows, where a token's row lies, and attention in 64 bits.  Written from the
definitions in include/scalekv.h; shares no code with the library."""
import numpy as np


def to_bf16(x):
    """float32 values rounded to bfloat16 (half to even), as float32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    nan = np.isnan(x)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)
    return np.where(nan, np.float32(np.nan), r)


def quantise(x):
    """[.., d] float32 -> (codes [.., d] int8, scales [..] float32): s = max|x| / 127, codes x / s half to even, both in fp32; a row
    with an infinity or a NaN has s = NaN and codes 0."""
    x = np.asarray(x, np.float32)
    fine = np.isfinite(x).all(-1)
    safe = np.where(fine[..., None], x, np.float32(0))
    s = (np.abs(safe).max(-1) / np.float32(127)).astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.rint((safe / s[..., None]).astype(np.float32))
    codes = np.where((s > 0)[..., None], np.clip(q, -127, 127), 0).astype(np.int8)
    return codes, np.where(fine, s, np.float32(np.nan))


def stored(x, store):
    """What the cache gives back for rows x, in fp32 (codes) or as the bf16 values."""
    if store == "bf16":
        return to_bf16(x)
    codes, s = quantise(x)
    return codes.astype(np.float32) * s[..., None]


def visible(n_new, length, causal, window, n_sink):
    """[n_new, length] bool: which positions the new tokens' queries see."""
    p = (length - n_new + np.arange(n_new))[:, None]
    j = np.arange(length)[None, :]
    seen = np.ones((n_new, length), bool)
    if causal:
        seen &= j <= p
    if window:
        seen &= (j > p - window) | (j < n_sink)
    return seen


def attend(q, k, v, seen, scale):
    """q [n, d], k and v [L, d], seen [n, L] in 64 bits -> O [n, d], lse [n], A [n, d] = sum of p |v| (what errors of p scale with) and
    Y [n] = the largest scale * sum |q_i k_i| over the keys seen (what errors of a product scale with)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, d = q.shape
    O, A, lse, Y = np.zeros((n, d)), np.zeros((n, d)), np.full(n, -np.inf), np.zeros(n)
    for i in range(n):
        at = seen[i]
        if not at.any():
            continue
        y = scale * (k[at] @ q[i])
        Y[i] = scale * (np.abs(k[at]) @ np.abs(q[i])).max()
        m = y.max()
        e = np.exp(y - m)
        lse[i] = m + np.log(e.sum())
        p = e / e.sum()
        O[i], A[i] = p @ v[at], p @ np.abs(v[at])
    return O, lse, A, Y


def turned(x, positions, axis, frequency, adjacent):
    """x [n, heads, d] in 64 bits with pair i turned by positions[axis[i]] * frequency[i] (positions [axes, n]), and [n, heads, d] |a| + |b| of every
    turning value's pair (what errors of an angle scale with)."""
    y, A, n = np.array(x, np.float64), np.zeros(x.shape), len(axis)
    for i in range(n):
        u, v = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
        f = np.asarray(positions[axis[i]], np.float64) * frequency[i]
        c, s = np.cos(f)[:, None], np.sin(f)[:, None]
        a, b = x[..., u].astype(np.float64), x[..., v].astype(np.float64)
        y[..., u], y[..., v] = a * c - b * s, a * s + b * c
        A[..., u] = A[..., v] = np.abs(a) + np.abs(b)
    return y, A


def draft_visible(sees, length):
    """[n_new, length] bool: new token i sees all that was there before, and of the new tokens those of sees[i]."""
    n = len(sees)
    seen = np.zeros((n, length), bool)
    for i, js in enumerate(sees):
        seen[i, :max(length - n, 0)] = True
        for j in js:
            if length - n + j >= 0:
                seen[i, length - n + j] = True
    return seen


def draft_bits(sees, words):
    """[n_new, words] int32: bit j mod 32 of word j / 32 is set for every j of sees[i]."""
    bits = np.zeros((len(sees), words), np.uint32)
    for i, js in enumerate(sees):
        for j in js:
            bits[i, j // 32] |= np.uint32(1 << (j % 32))
    return bits.view(np.int32)


def attention_got(q, k, lse, seen, scale):
    """Rows q [n, d], their log-sum-exps, keys k [L, d], seen [n, L] in 64 bits -> what every key gets, sum over rows of p = exp(scale q.k - lse) [L], and
    the sums of p Y with Y = scale sum |q_i k_i|, and of p (1 + |lse| + |scale q.k|) (what errors of a product, and of an exponent, scale with)."""
    q, k = np.asarray(q, np.float64), np.asarray(k, np.float64)
    lse = np.asarray(lse, np.float64)[:, None]
    y, Y = scale * (q @ k.T), scale * (np.abs(q) @ np.abs(k).T)
    with np.errstate(over="ignore", invalid="ignore"):
        p = np.where(seen & (lse != -np.inf), np.exp(y - np.where(lse == -np.inf, 0, lse)), 0.0)
    finite = np.where(np.isfinite(lse), np.abs(lse), 0)
    return p.sum(0), (p * Y).sum(0), (p * (1 + finite + np.abs(y))).sum(0)


def stays(weights, keep, n_sink, n_recent):
    """Positions of weights [L] that stay, ascending: min(keep, L) of them, the first n_sink, the last n_recent as far as there is room, the heaviest of the rest; of
    equal weights the first, a NaN is -inf."""
    L = len(weights)
    k = min(keep, L)
    sinks = min(n_sink, k)
    recent = min(n_recent, k - sinks)
    w = np.where(np.isnan(weights), -np.inf, weights)
    middle = sorted(range(sinks, L - recent), key=lambda j: (-w[j], j))[:k - sinks - recent]
    return np.array(list(range(sinks)) + sorted(middle) + list(range(L - recent, L)), np.int64)
