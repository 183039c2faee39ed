"""The oracle of the 8-bit serving operators against values worked out by hand and against its own definition."""
import numpy as np
import pytest

from oracle import qcfg_oracle as orc
from oracle import serve_oracle as so


def test_token_codes_are_the_per_row_codes():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((9, 33)).astype(np.float32)
    x[3] = 0
    for bits in range(2, 9):
        s, inv = orc.scales_from_absmax(orc.absmax(x, orc.PER_ROW), bits)
        q, got = so.quantize_tokens(x, bits)
        np.testing.assert_array_equal(q, orc.quantize(x, inv[:, None], bits))
        np.testing.assert_array_equal(got, s)


def test_nonfinite_and_tiny_values():
    x = np.array([[1.0, np.nan, -2.0, np.inf], [1e-38, 0.0, -1e-38, 5e-39]], np.float32)
    q, s = so.quantize_tokens(x)
    np.testing.assert_array_equal(q[0], [64, 0, -127, 0])      # 63.5 rounds to the even 64
    assert s[0] == np.float32(2) / np.float32(127)
    # 127 / 1e-38 is Inf: zeros stay zero, the rest is clamped
    np.testing.assert_array_equal(q[1], [127, 0, -127, 127])


def test_pages_of_a_small_pool():
    p = so.Pool(6, 4, 5, 4)
    assert p.extend([0, -1, 1], [5, 9, 4])
    assert p.table[0] == [0, 1] and p.table[1] == [2] and p.lens[:2] == [5, 4] and p.refs == [1, 1, 1, 0, 0, 0]
    assert not p.extend([0, 0], [1, 1]) and not p.extend([2], [17]) and not p.extend([2, 3], [12, 4])
    assert p.fork([0, 1], [2, 3]) == ([1, -1], [3, -1])
    assert p.table[2] == [0, 3] and p.table[3] == [2] and p.refs == [2, 1, 2, 1, 0, 0]
    assert p.fork([0], [1]) is None and p.fork([0, 0], [4, 4]) is None
    p.free([0, 0, -1])
    assert p.refs == [1, 0, 2, 1, 0, 0] and p.lens[0] == 0
    assert p.compact() == [0, -1, 2, 1, -1, -1]
    assert p.table == [[], [2], [0, 1], [2], []] and p.refs == [1, 1, 2, 0, 0, 0]


def test_a_larger_token_moves_the_page_to_a_new_grid():
    p = so.Pool(2, 16, 1, 2)
    c = so.Cache(p, 1, 16)
    a = np.full((1, 1, 16), 1.0, np.float32)
    assert p.extend([0], [1])
    c.append(a, a, [0], [0, 1])
    assert p.extend([0], [1])
    c.append(4 * a, a, [0], [0, 1])
    k, v = c.values(0)
    # 127 * (1/4) = 31.75 -> 32 on the grid of 4/127
    np.testing.assert_allclose(k[:, 0, 0], [32 * np.float32(4 / 127), 127 * np.float32(4 / 127)], rtol=1e-6)
    np.testing.assert_allclose(v[:, 0, 0], [1, 1], rtol=1e-6)


@pytest.mark.parametrize("causal,window,want", [(True, 0, [[0, 0, 0], [1, 0, 0], [1, 1, 0], [1, 1, 1]]), (False, 0, [[0, 0, 0]] + 3 * [[1, 1, 1]]),
                                                (True, 2, [[0, 0, 0], [1, 0, 0], [1, 1, 0], [0, 1, 1]])])
def test_what_a_row_sees(causal, window, want):
    np.testing.assert_array_equal(so.seen(4, 3, causal, window), np.array(want, bool))


def test_attention_of_one_token_is_its_value():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 4, 16)), rng.standard_normal((1, 2, 16)), rng.standard_normal((1, 2, 16))
    out, _, _ = so.attention(q, k, v, 0.25)
    assert not out[0].any()                                    # the first row stands before the only token
    np.testing.assert_allclose(out[1], v[0][[0, 0, 1, 1]], rtol=1e-12)
