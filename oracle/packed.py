"""Oracle of the operators on packed sequences and continued turns, plain numpy in fp64: the convolution tap by tap, the recurrence token by
token, attention query by query, rotations as complex numbers.  Shares no code with the library.

Where a result is a sum of terms that a kernel may round one by one, the sum of the terms' absolute values comes with it: what a relative error of
each term is multiplied by.
"""
import math

import numpy as np


def conv(zx, d_inner, conv_w, conv_b, dt_bias, starts, window):
    """Pre-scan step of packed rows.  Returns (u [rows, channels] after SiLU, sum of absolute terms, dt [rows, H], windows out
    [n_seq, W-1, channels]); rows of no sequence are NaN.  window None: zeros."""
    zx = np.asarray(zx, dtype=np.float64)
    ch, W = conv_w.shape
    H, n_seq = len(dt_bias), len(starts) - 1
    u, mag, dt = (np.full((len(zx), m), np.nan) for m in (ch, ch, H))
    out = np.zeros((n_seq, W - 1, ch))
    for s in range(n_seq):
        a, b = starts[s], starts[s + 1]
        line = [np.zeros(ch) if window is None else np.asarray(window[s][j], dtype=np.float64) for j in range(W - 1)]
        line += [zx[t, d_inner:d_inner + ch] for t in range(a, b)]
        for t in range(a, b):
            taps = [conv_w[:, j].astype(np.float64) * line[t - a + j] for j in range(W)]
            acc = conv_b.astype(np.float64) + sum(taps)
            u[t] = acc / (1.0 + np.exp(-acc))
            mag[t] = np.abs(conv_b) + sum(np.abs(x) for x in taps)
            raw = zx[t, d_inner + ch:] + dt_bias
            dt[t] = np.log1p(np.exp(-np.abs(raw))) + np.maximum(raw, 0.0)
        out[s] = line[len(line) - (W - 1):]
    return u, mag, dt, out


def scan(x, dt, A, B, C, D, starts, state):
    """The recurrence of packed sequences.  Returns (y [rows, H, p], its sum of absolute terms, final states [n_seq, H, p, n], theirs);
    rows of no sequence are NaN.  state None: zeros."""
    x, dt, A, B, C = (np.asarray(a, dtype=np.float64) for a in (x, dt, A, B, C))
    rows, H, p = x.shape
    G, n = B.shape[1:]
    n_seq = len(starts) - 1
    y, ymag = np.full(x.shape, np.nan), np.full(x.shape, np.nan)
    S = np.zeros((n_seq, H, p, n)) if state is None else np.array(state, dtype=np.float64)
    M = np.abs(S)
    for s in range(n_seq):
        for t in range(starts[s], starts[s + 1]):
            a = np.exp(dt[t] * A)[:, None, None]
            b, c = np.repeat(B[t], H // G, axis=0)[:, None, :], np.repeat(C[t], H // G, axis=0)[:, None, :]
            term = (dt[t][:, None] * x[t])[..., None] * b
            S[s] = a * S[s] + term
            M[s] = a * M[s] + np.abs(term)
            y[t], ymag[t] = (S[s] * c).sum(-1), (M[s] * np.abs(c)).sum(-1)
            if D is not None:
                skip = np.asarray(D, dtype=np.float64)[:, None] * x[t]
                y[t] += skip
                ymag[t] += np.abs(skip)
    return y, ymag, S, M


def attention(q, k, v, q_starts, k_starts, scale):
    """Causal attention of packed sequences.  Returns (o [rows_q, Hq, d], sum_j p_j |v_j|, the largest sum_c |q_c k_c| scale over the
    pairs seen); rows of no sequence are NaN, rows without keys zero."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    Hq, Hkv = q.shape[1], k.shape[1]
    o, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    largest = 0.0
    for s in range(len(q_starts) - 1):
        lq, lk = q_starts[s + 1] - q_starts[s], k_starts[s + 1] - k_starts[s]
        for i in range(lq):
            t, m = q_starts[s] + i, lk - lq + i + 1
            if m <= 0:
                o[t] = mag[t] = 0.0
                continue
            K, V = k[k_starts[s]:k_starts[s] + m], v[k_starts[s]:k_starts[s] + m]
            for h in range(Hq):
                g = h // (Hq // Hkv)
                z = K[:, g] @ q[t, h] * scale
                w = np.exp(z - z.max())
                w /= w.sum()
                o[t, h], mag[t, h] = w @ V[:, g], w @ np.abs(V[:, g])
                largest = max(largest, (np.abs(K[:, g]) @ np.abs(q[t, h])).max() * scale)
    return o, mag, largest


def rope_frequencies(theta, rot_dim, scaling="none", factor=1.0, trained_len=0, turns=(1.0, 32.0)):
    f = []
    for i in range(rot_dim // 2):
        v = math.exp(-2.0 * i / rot_dim * math.log(theta))
        if scaling == "linear":
            v /= factor
        elif scaling == "banded":
            g = min(1.0, max(0.0, (trained_len * v / (2.0 * math.pi) - turns[0]) / (turns[1] - turns[0])))
            v = g * v + (1.0 - g) * v / factor
        f.append(v)
    return np.array(f)


def rope(qkv, positions, Hq, Hkv, d, frequencies, layout="half", amplitude=1.0):
    """(q, k, v) of the rows, the pairs of the first 2 len(frequencies) elements of q and k heads turned.  Angles are reduced with more than 64
    bits: position times turns in rational arithmetic of the frequency's own 64-bit value."""
    rows = np.array(qkv, dtype=np.float64).reshape(len(qkv), Hq + 2 * Hkv, d)
    half = len(frequencies)
    first, second = (np.arange(half), np.arange(half) + half) if layout == "half" else (2 * np.arange(half), 2 * np.arange(half) + 1)
    out = rows.copy()
    for r, pos in enumerate(positions):
        angle = np.array([float(np.fmod(np.longdouble(int(pos)) * np.longdouble(f), 2 * np.longdouble("3.14159265358979323846264338327950288"))) for f in frequencies])
        z = (rows[r, :Hq + Hkv][:, first] + 1j * rows[r, :Hq + Hkv][:, second]) * (amplitude * np.exp(1j * angle))
        out[r, :Hq + Hkv][:, first], out[r, :Hq + Hkv][:, second] = z.real, z.imag
    return out[:, :Hq], out[:, Hq:Hq + Hkv], out[:, Hq + Hkv:]
