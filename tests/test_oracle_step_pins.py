"""The definitions of oracle/step_oracle.py against hand-made values and other formulations (CPU)."""
import cmath
import math

import numpy as np
import pytest

from oracle import step_oracle as S


def test_page_table_by_hand():
    # 17 tokens and 3 spare: two pages, one held already; an empty segment keeps its page; a new one gets two.
    off, pages = S.page_table([17, 0, 30], 3, [0, 1, 2], [7, 8], [20, 21, 22, 23])
    assert off.tolist() == [0, 2, 3, 6] and pages.tolist() == [7, 20, 8, 21, 22, 23]
    off, pages = S.page_table([17, 16], 0, [], [], [5])
    assert off.tolist() == [0, 2, 3] and pages.tolist() == [5, -1, -1]
    off, pages = S.page_table([1], 0, [0, 3], [4, 5, 6], [9])            # more pages than it needs stay
    assert off.tolist() == [0, 3] and pages.tolist() == [4, 5, 6]


def graph():
    """Two branches over a prompt of 20 tokens; pages 5, 3 | 4 | 1."""
    return S.Graph([20, 2, 16], [0, 2, 3, 4], [5, 3, 4, 1], [0, 2, 4], [0, 1, 0, 2], 6)


def test_slot_map_by_hand():
    off, words, positions, branches = S.slot_map(graph(), [2, 1], 4)
    assert off.tolist() == [0, 2, 3]
    assert words.tolist() == [64, 65, 31, -1] and positions.tolist() == [20, 21, 35, -1]
    assert branches.tolist() == [0, 0, 1, -1]
    # More new tokens than the segment has: those before its start are padding.
    off, words, positions, branches = S.slot_map(graph(), [3, 0], 3)
    assert words.tolist() == [-1, 64, 65] and positions.tolist() == [-1, 20, 21] and branches.tolist() == [-1, 0, 0]


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, pos, freq = rng.standard_normal((3, 2, 8)), np.array([0, 5, 1000]), np.array([1.0, 0.1, 0.01])
    y, reach = S.norm_rotate(x, pos, freq, interleaved, None, 0.0, 1.0)
    for n in range(3):
        for i in range(3):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 3)
            for h in range(2):
                z = complex(x[n, h, a], x[n, h, b]) * cmath.exp(1j * float(pos[n]) * float(freq[i]))
                assert abs(y[n, h, a] - z.real) < 1e-12 and abs(y[n, h, b] - z.imag) < 1e-12
    np.testing.assert_array_equal(y[..., 6:], x[..., 6:])
    # Lengths of pairs stay, products depend on the distance of positions alone.
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    q, k = S.norm_rotate(x[:1], [7], freq, interleaved, None, 0.0, 1.0)[0], S.norm_rotate(x[1:2], [3], freq, interleaved, None, 0.0, 1.0)[0]
    q2, k2 = S.norm_rotate(x[:1], [104], freq, interleaved, None, 0.0, 1.0)[0], S.norm_rotate(x[1:2], [100], freq, interleaved, None, 0.0, 1.0)[0]
    assert np.allclose((q * k).sum(-1), (q2 * k2).sum(-1))


def test_norm_by_hand():
    y, _ = S.norm_rotate(np.array([[[3.0, 4.0]]]), [9], [], False, np.array([2.0, 1.0]), 0.0, 1.0)
    r = math.sqrt(12.5)
    assert np.allclose(y, [[[6 / r, 4 / r]]])
    # A multiple of a row has its norm.
    x = np.random.default_rng(2).standard_normal((1, 1, 16))
    one, ten = (S.norm_rotate(f * x, [0], [], False, np.ones(16), 0.0, 1.0)[0] for f in (1, 10))
    assert np.allclose(one, ten) and np.allclose((one ** 2).mean(), 1.0)


def test_context_and_rules_by_hand():
    ids = np.full(96, -1)
    ids[5 * 16:5 * 16 + 16] = 2                           # the prompt's first page
    ids[[48, 49, 50, 51]] = [3, 3, 0, -1]
    ids[[64, 65]] = [4, 3]
    g = graph()
    assert S.context(g, 0, None, ids, 1) == [(2, True)] * 16 + [(3, True), (3, True), (0, True), (-1, True), (4, False), (3, False)]
    assert S.context(g, 0, 20, ids, 1)[-1] == (4, False) and len(S.context(g, 0, 3, ids, 1)) == 4
    z, _ = S.logits_row([1.0, -2.0, 3.0, -4.0, 6.0], S.context(g, 0, None, ids, 1), rep=2.0, freq=0.5, pres=0.25, temp=2.0,
                        bias=[(1, 5.0), (1, 1.0)], allowed=np.array([1, 1, 0, 1, 1], bool))
    # prompt only: 0, 2; said: 3 (also in the prompt), 4
    assert z.tolist() == [0.25, 2.0, -math.inf, (-8 - 0.75) / 2, (3 - 0.75) / 2]
