"""Oracle of the decode-side operators: the 4-bit key/value cache and the single-token Mamba-2 step, plain numpy.

The quantisation is defined in fp32 arithmetic and is bit-exact; everything else is fp64.  Shares no code with the
library: rows are packed and unpacked here element by element from the documented order.
"""
import numpy as np


def bf16_floor(x):
    """Largest bf16 value <= x, for finite fp32 x, as fp32."""
    bits = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    up = (bits & np.uint32(0xFFFF0000)) + np.where((bits >> 31 == 1) & (bits & 0xFFFF != 0), np.uint32(0x10000), np.uint32(0))
    return up.astype(np.uint32).view(np.float32)


def bf16_round(x):
    """Nearest bf16 value (ties to even) of finite fp32 x, as fp32."""
    bits = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def kv4_quantise(x, group):
    """(codes uint8 [..., d], zero fp32, scale fp32 [..., d / group]) of fp32 rows; a group with a value that is not finite
    gets a NaN scale."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    g = x.reshape(*x.shape[:-1], -1, group)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], np.float32(0), g)
    with np.errstate(over="ignore"):
        zero = bf16_floor(g.min(-1))
        span = (g.max(-1) - zero) * (np.float32(1) / np.float32(15))
        over = ~np.isfinite(span)
        scale = bf16_round(np.where(over, np.float32(0), span))
        over |= ~np.isfinite(scale)
        scale[over] = 0
        step = np.where(scale > 0, scale, np.float32(1))[..., None]
        code = np.where(scale[..., None] > 0, np.clip(np.rint((g - zero[..., None]) / step), 0, 15), 0).astype(np.uint8)
    bad |= over
    code[bad] = 0
    scale = np.where(bad, np.float32(np.nan), scale)
    return code.reshape(x.shape), zero, scale


def kv4_values(code, zero, scale, group):
    """fp64 values the codes stand for."""
    g = code.reshape(*code.shape[:-1], -1, group).astype(np.float64)
    return (zero[..., None].astype(np.float64) + scale[..., None].astype(np.float64) * g).reshape(code.shape)


def kv4_element_nibble(d, keys):
    """For every element of a row, the index of its nibble in the packed row (nibble 2i is the low half of byte i)."""
    ng = d // 32
    at = np.empty(d, dtype=np.int64)
    for e in range(d):
        g, w = divmod(e, 32)
        at[e] = ((w // 8) * ng + g) * 8 + w % 8 if keys else ((w // 4) * ng + g) * 4 + w % 4
    return at


def kv4_pack(code, keys):
    d = code.shape[-1]
    nib = np.zeros(code.shape, dtype=np.uint8)
    nib[..., kv4_element_nibble(d, keys)] = code
    return nib[..., 0::2] | (nib[..., 1::2] << 4)


def kv4_unpack(packed, keys):
    nib = np.stack((packed & 15, packed >> 4), -1).reshape(*packed.shape[:-1], -1)
    return nib[..., kv4_element_nibble(nib.shape[-1], keys)]


def kv4_words(zero, scale):
    """32-bit words: bf16 scale in the high half, bf16 zero in the low half."""
    s = np.where(np.isnan(scale), np.uint32(0x7FFF0000), scale.view(np.uint32) & np.uint32(0xFFFF0000))
    z = np.where(np.isnan(scale), np.uint32(0), zero.view(np.uint32) >> 16)
    return (s | z).astype(np.uint32)


def kv4_attention(q, k, v, scale):
    """q [n_q, Hq, d] of one sequence's newest tokens; k, v [Hkv, len, d] the values in its cache.  Returns (o [n_q, Hq, d],
    drawn [Hkv, len]: the softmax weights that fell on each row)."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    n_q, Hq, d = q.shape
    Hkv, n, _ = k.shape
    o, drawn = np.zeros(q.shape), np.zeros((Hkv, n))
    for i in range(n_q):
        m = n - n_q + i + 1
        if m <= 0:
            continue
        for hq in range(Hq):
            h = hq // (Hq // Hkv)
            s = k[h, :m] @ q[i, hq] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o[i, hq] = p @ v[h, :m]
            drawn[h, :m] += p
    return o, drawn


def kv4_evict(weight, n, keep, n_recent, n_evictable=None):
    """weight [Hkv, cap] of one sequence with n rows: the ascending indices of the min(n, keep) rows that stay."""
    big = np.finfo(np.float32).max
    score = np.zeros(n)
    for h in range(weight.shape[0]):
        score = score + weight[h, :n].astype(np.float64)
    with np.errstate(over="ignore"):
        score = score.astype(np.float32)
    score = np.where(np.isnan(score), -big, np.clip(score, -big, big))
    first = n - n_recent if n_evictable is None else min(n - n_recent, n_evictable)
    first = max(first, n - keep, 0)
    ranked = sorted(range(first), key=lambda t: (-score[t], t))
    return np.array(sorted(ranked[:max(0, min(n, keep) - (n - first))]) + list(range(first, n)), dtype=np.int32)


def mamba2_step(x, dt, A, B, C, state, D=None):
    """T tokens of the recurrence of one sequence from `state` [H, p, n]: (y [T, H, p], state after the last token)."""
    T, H, p = x.shape
    per = H // B.shape[1]
    S, y = np.array(state, dtype=np.float64), np.zeros((T, H, p))
    for t in range(T):
        for h in range(H):
            b, c = B[t, h // per].astype(np.float64), C[t, h // per].astype(np.float64)
            S[h] = np.exp(float(dt[t, h]) * float(A[h])) * S[h] + np.outer(float(dt[t, h]) * x[t, h].astype(np.float64), b)
            y[t, h] = S[h] @ c + (float(D[h]) * x[t, h] if D is not None else 0.0)
    return y, S
