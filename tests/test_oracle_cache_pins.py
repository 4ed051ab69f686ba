"""Pins of the compressed-cache oracle: MXFP4 rounding and page layout, attention mass, eviction."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as C
from oracle import graphattn_oracle as O
from paper_2606_18954_amd import workloads as W


def test_block_exponents():
    def e(top):
        x = np.zeros(32)
        x[7] = -top
        return C.block_exponent(x)
    assert [e(4.0), e(6.0), e(6.99), e(7.0), e(8.0)] == [0, 0, 0, 1, 1]
    assert [e(1.0), e(0.5), e(3.4)] == [-2, -3, -1]
    assert e(0.0) == -125 and e(1e-40) == -125 and e(3.3e38) == 125
    assert e(math.inf) is None and e(math.nan) is None


def test_codes_and_ties():
    ys = [0.0, 0.25, 0.26, 0.5, 0.75, 1.25, 1.26, 1.75, 2.5, 3.5, 4.9, 5.0, 5.1, 6.0, 7.0, 100.0]
    want = [0, 0, 1, 1, 2, 2, 3, 4, 4, 6, 6, 6, 7, 7, 7, 7]
    assert [C.nearest_code(y) for y in ys] == want
    assert [C.nearest_code(-y) for y in ys] == [w + 8 for w in want]


def test_rounding_error_is_bounded():
    """The widest step of the codes is 2 x 2^e, and the top lies below 7 x 2^e where the largest value is
    6 x 2^e: no value is off by more than 2^e, and none changes its sign."""
    rng = np.random.default_rng(3)
    for _ in range(200):
        x = rng.standard_normal(32) * 10.0 ** rng.uniform(-6, 6)
        codes, byte = C.quantise_block(x)
        got = np.array([C.code_value(c, byte) for c in codes])
        assert np.abs(got - x).max() <= 2.0 ** (byte - 127)
        assert np.abs(x).max() < 7 * 2.0 ** (byte - 127)
        assert np.array_equal(np.sign(got)[np.abs(got) > 0], np.sign(x)[np.abs(got) > 0])


@pytest.mark.parametrize("D", [64, 128])
def test_places_are_a_partition_of_the_page(D):
    code = {(v, t, c): C.code_place(t, c, D, v) for v in (False, True) for t in range(16)
            for c in range(D)}
    assert len(set(code.values())) == 32 * D
    scale = {(v, t, b): C.scale_place(t, 32 * b, D, v) for v in (False, True) for t in range(16)
             for b in range(D // 32)}
    assert len(set(scale.values())) == D
    used = {b for b, _ in code.values()} | set(scale.values())
    assert used == set(range(17 * D))


def test_append_and_values_round_trip():
    rng = np.random.default_rng(5)
    pool = rng.integers(0, 256, (3, 2, 17 * 64)).astype(np.uint8)
    k, v = rng.standard_normal((4, 2, 64)), rng.standard_normal((4, 2, 64))
    words = [5, -1, 40, 48]                              # the last lies outside the pool
    out = C.append(pool, k, v, words)
    vals = C.pool_values(out)
    for j, w in ((0, 5), (2, 40)):
        for h in range(2):
            for x, i in ((k, 0), (v, 1)):
                for b in (0, 32):
                    codes, byte = C.quantise_block(x[j, h, b:b + 32])
                    want = [C.code_value(c, byte) for c in codes]
                    assert np.array_equal(vals[w // 16, h, i, w % 16, b:b + 32], want)
    # Nothing else changed.
    before, after = C.pool_values(pool), vals
    for w in range(48):
        if w not in (5, 40):
            assert np.array_equal(before[w // 16, :, :, w % 16], after[w // 16, :, :, w % 16],
                                  equal_nan=True)


def _small(counts=None):
    rng = np.random.default_rng(9)
    g = W.assemble_graph([20, 7, 33, 4], [[0, 1], [0, 2], [0, 3]], 4, slack_pages=1)
    values = rng.standard_normal((g.num_pages, 2, 2, 16, 64))
    rows = 3 if counts is None else sum(counts)
    return g, values, rng.standard_normal((rows, 4, 64))


def test_attention_agrees_with_the_textbook_oracle():
    g, values, q = _small()
    q32, v32 = q.astype(np.float32), values.astype(np.float32)
    out, lse, spread, _ = C.attention(q32.astype(float), v32.astype(float), g, 4, 2)
    oo, ol = O.decode(q32, v32, g.seg_len, g.seg_page_offsets, g.seg_pages, g.path_offsets,
                      g.path_segs, 4, 2, 64, "f32")
    assert np.abs(out - oo).max() < 1e-12 and np.abs(lse - ol).max() < 1e-12
    assert (spread >= np.abs(out) - 1e-12).all()


@pytest.mark.parametrize("counts", [None, [3, 5, 4]])
def test_masses_add_up_to_the_rows(counts):
    """Softmax weights of a row add to one: with the rows' own lse, the new mass of all slots is the
    number of (row, head) pairs, and the earlier mass comes in by its factor."""
    g, values, q = _small(counts)
    lse = C.attention(q, values, g, 4, 2, counts)[1]
    zero = np.zeros(16 * g.num_pages)
    m = C.mass(q, values, g, lse, 4, 2, zero, 0.5, counts)
    assert abs(np.nansum(m) - 4 * len(q)) < 1e-9
    assert np.isfinite(m).sum() == g.unique_tokens()
    m2 = C.mass(q, values, g, lse, 4, 2, np.ones(16 * g.num_pages), 0.5, counts)
    assert np.nanmax(np.abs(m2 - m - 0.5)) < 1e-12
    lse[1, 2] = math.inf                                 # a row that counts for nothing
    assert abs(np.nansum(C.mass(q, values, g, lse, 4, 2, zero, 0.5, counts))
               - (4 * len(q) - 1)) < 1e-9


def test_keep_tokens():
    w = [5.0, 1.0, 3.0, 3.0, 9.0, 3.0, 0.0, 2.0]
    assert C.keep_tokens(w, 3, 0, 0) == [0, 2, 4]        # ties to the lower position
    assert C.keep_tokens(w, 4, 2, 1) == [0, 1, 4, 7]     # protected ones first
    assert C.keep_tokens(w, 8, 0, 0) == list(range(8))
    assert C.keep_tokens(w, 0, 0, 0) == []
    assert C.keep_tokens([1.0, math.nan, math.inf], 1, 0, 0) == [1]
    assert C.keep_tokens([0.0, -0.0, -1.0], 2, 0, 0) == [0, 1]


def test_evict_select_words():
    g = W.assemble_graph([20, 3], [[0, 1]], 8)
    m = np.arange(16.0 * g.num_pages)
    pos, words = C.evict_select(m, g.seg_len, g.seg_page_offsets, g.seg_pages, [2, 3], 1, 1)
    assert list(pos) == [0, 19, 0, 1, 2]
    p = g.seg_pages
    assert list(words) == [16 * p[0], 16 * p[1] + 3, 16 * p[2], 16 * p[2] + 1, 16 * p[2] + 2]
