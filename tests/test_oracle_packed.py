"""Pins of the packed-sequence oracle to closed forms and to the oracle of the unpacked operators."""
import math

import numpy as np
import pytest

import oracle
from oracle import packed


def test_convolution_of_one_sequence_is_a_correlation_and_windows_continue_it():
    g = np.random.default_rng(0)
    ch, W, H, T = 6, 4, 2, 9
    zx = g.standard_normal((T, 3 + ch + H))
    w, b, bias = g.standard_normal((ch, W)), g.standard_normal(ch), g.standard_normal(H)
    u, mag, dt, win = packed.conv(zx, 3, w, b, bias, [0, T], None)
    for c in range(ch):
        acc = np.convolve(zx[:, 3 + c], w[c, ::-1])[:T] + b[c]
        assert np.allclose(u[:, c], acc / (1 + np.exp(-acc)), rtol=1e-12, atol=1e-14)
    assert np.array_equal(win[0], zx[T - 3:, 3:3 + ch]) and (mag > 0).all()
    assert np.allclose(np.exp(dt), 1 + np.exp(zx[:, 3 + ch:] + bias))
    cut = 2                                                # two turns, the first shorter than the window
    u1, _, _, w1 = packed.conv(zx[:cut], 3, w, b, bias, [0, cut], None)
    u2, _, _, w2 = packed.conv(zx[cut:], 3, w, b, bias, [0, T - cut], w1)
    assert np.allclose(np.concatenate((u1, u2)), u) and np.array_equal(w2, win)
    _, _, _, w3 = packed.conv(zx, 3, w, b, bias, [4, 4], w1)
    assert np.array_equal(w3, w1)                          # an empty sequence hands its window on


def test_scan_of_packed_sequences_is_the_recurrence_of_each():
    g = np.random.default_rng(1)
    T, H, p, G, n = 11, 4, 3, 2, 5
    x, B, C = g.standard_normal((T, H, p)), g.standard_normal((T, G, n)), g.standard_normal((T, G, n))
    dt, A, D = 0.1 * g.random((T, H)), -g.random(H), g.standard_normal(H)
    y, ymag, S, M = packed.scan(x, dt, A, B, C, None, [0, 4, 4, 10], None)
    for a, b, s in ((0, 4, 0), (4, 10, 2)):
        ref, state = oracle.mamba2_recurrence(x[a:b], dt[a:b], A, B[a:b], C[a:b])
        assert np.allclose(y[a:b], ref) and np.allclose(S[s], state)
    assert np.isnan(y[10]).all() and (S[1] == 0).all() and (np.abs(S) <= M).all()
    y1, _, S1, _ = packed.scan(x[:4], dt[:4], A, B[:4], C[:4], D, [0, 4], None)
    y2, _, S2, _ = packed.scan(x[4:], dt[4:], A, B[4:], C[4:], D, [0, 7], S1)
    yy, yymag, SS, _ = packed.scan(x, dt, A, B, C, D, [0, T], None)
    assert np.allclose(np.concatenate((y1, y2)), yy) and np.allclose(S2, SS) and (np.abs(yy) <= yymag + 1e-12).all()


def test_attention_of_equal_scores_is_a_mean_and_hidden_keys_do_not_count():
    v = np.arange(12.0).reshape(6, 1, 2)
    q, k = np.zeros((4, 2, 2)), np.zeros((6, 1, 2))
    o, mag, largest = packed.attention(q, k, v, [0, 1, 1, 4], [0, 4, 4, 6], 1.0)
    assert np.allclose(o[0, 0], v[:4, 0].mean(0)) and largest == 0.0
    assert (o[1] == 0).all()                               # three queries, two keys: the first sees none
    assert np.allclose(o[2, 1], v[4, 0]) and np.allclose(o[3, 0], v[4:6, 0].mean(0)) and np.allclose(mag, np.abs(o))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_turns_pairs_by_their_angle(layout):
    f = packed.rope_frequencies(100.0, 4)
    assert np.allclose(f, [1.0, 0.1])
    rows = np.zeros((1, 3 * 6))
    rows[0, [0, 6, 12]] = 1.0                              # the first element of each head
    q, k, v = packed.rope(rows, [2], 1, 1, 6, f, layout, 3.0)
    other = 2 if layout == "half" else 1
    want = np.zeros(6)
    want[0], want[other] = 3 * math.cos(2.0), 3 * math.sin(2.0)
    assert np.allclose(q[0, 0], want) and np.allclose(k[0, 0], want) and np.array_equal(v[0, 0], [1, 0, 0, 0, 0, 0])


def test_stretched_frequencies():
    plain = packed.rope_frequencies(1e6, 64)
    assert np.allclose(packed.rope_frequencies(1e6, 64, "linear", 4.0), plain / 4)
    banded = packed.rope_frequencies(1e6, 64, "banded", 4.0, 32768, (1.0, 32.0))
    turns = 32768 * plain / (2 * math.pi)
    assert np.allclose(banded[turns >= 32], plain[turns >= 32]) and np.allclose(banded[turns <= 1], plain[turns <= 1] / 4)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (banded[between] < plain[between]).all() and (banded[between] > plain[between] / 4).all()
