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
