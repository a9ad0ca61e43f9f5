"""Pins of oracle/window.py: the plain attention of oracle/transformer.py, cases worked by hand, properties of the rounding."""
import numpy as np
import pytest

from oracle import transformer as T
from oracle import window as W


def test_visible_by_hand():
    want = {0: [0], 1: [0, 1], 2: [0, 1, 2], 3: [0, 2, 3], 5: [0, 4, 5]}
    for i, keys in want.items():
        assert np.flatnonzero(W.visible([i], 7, 2, 1)[0]).tolist() == keys


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (3, 2), (5, 50)])
def test_number_of_visible_keys(window, sinks):
    n = 20
    got = W.visible(np.arange(n), n, window, sinks).sum(1)
    assert got.tolist() == [min(i + 1, window) + min(sinks, max(0, i + 1 - window)) for i in range(n)]


@pytest.mark.parametrize("window,sinks", [(9, 0), (100, 3), (4, 9)])
def test_all_visible_is_causal_attention(window, sinks):
    r = np.random.default_rng(0)
    q, k, v = r.normal(size=(9, 6, 8)), r.normal(size=(9, 3, 8)), r.normal(size=(9, 3, 8))
    np.testing.assert_allclose(W.attention(q, k, v, np.arange(9), window, sinks), T.attention(q, k, v, np.arange(9)), atol=1e-13)


def test_window_of_one_is_the_value_itself():
    r = np.random.default_rng(1)
    q, k, v = r.normal(size=(5, 2, 8)), r.normal(size=(5, 2, 8)), r.normal(size=(5, 2, 8))
    np.testing.assert_allclose(W.attention(q, k, v, np.arange(5), 1, 0), v, atol=0)


def test_window_is_attention_over_the_keys_it_leaves():
    """Position 7 with window 3 and 2 sinks: attention over the keys 0, 1, 5, 6, 7 alone; hidden ones may hold anything."""
    r = np.random.default_rng(2)
    q, k, v = r.normal(size=(1, 4, 8)), r.normal(size=(9, 2, 8)), r.normal(size=(9, 2, 8))
    at = [0, 1, 5, 6, 7]
    want = T.attention(q, k[at], v[at], np.array([4]))
    k[[2, 3, 4, 8]], v[[2, 3, 4, 8]] = np.nan, np.inf
    np.testing.assert_allclose(W.attention(q, k, v, [7], 3, 2), want, atol=1e-13)


def test_rounding_by_hand():
    """-1 .. 14 in steps of one: s = 1, c = 7, every value held; with 0.5 and 1.5 half way between two steps."""
    x = np.zeros(64)
    x[:16] = np.arange(-1, 15)
    x[16], x[17] = 0.5, 1.5
    codes, p = W.kv4_quantize(x)
    assert p[0].tolist() == [1.0, 7.0]
    assert codes[:16].tolist() == list(range(16))
    assert W.kv4_round(x)[:18].tolist() == list(range(-1, 15)) + [1.0, 1.0]       # u = -6.5 and -5.5: both to -6


def test_rounding_error_and_edges():
    r = np.random.default_rng(3)
    x = r.normal(size=(50, 128)).astype(np.float32)
    codes, p = W.kv4_quantize(x)
    s = np.repeat(p[..., 0].astype(np.float64), 64, -1)
    # inside the range of the steps half a step; s and c are rounded (2^-11 of themselves), which moves the ends by 8 |s| 2^-11 + |c| 2^-11
    assert (np.abs(W.kv4_values(codes, p) - x) <= s * (0.5 + 0.01) + 0.01 * s).all()
    assert set(np.unique(codes)) == set(range(16))
    np.testing.assert_array_equal(W.kv4_round(np.full(64, 0.1, np.float32)), np.float64(np.float16(0.1)))
    assert np.isnan(W.kv4_round(np.r_[np.ones(63), np.inf])).all()
    far = W.kv4_round(np.r_[np.ones(64), np.full(64, 70000.0)].astype(np.float32))
    assert (far[:64] == 1).all() and np.isnan(far[64:]).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_block_holds_every_value_in_a_place_of_its_own(hd):
    k_byte, k_bit, v_byte, v_bit, par = W.kv4_places(hd)
    nibbles = [set((b * 8 + s).flatten().tolist()) for b, s in ((k_byte, k_bit), (v_byte, v_bit))]
    assert nibbles[0] == set(range(0, 64 * hd, 4)) and nibbles[1] == set(range(64 * hd, 128 * hd, 4))
    assert set(par.flatten().tolist()) == set(range(16 * hd, 17 * hd, 4))
    r = np.random.default_rng(4)
    k, v = r.normal(size=(16, hd)).astype(np.float32), r.normal(size=(16, hd)).astype(np.float32)
    block = r.integers(0, 256, 18 * hd).astype(np.uint8)
    for t in r.permutation(16):
        W.kv4_write(block, t, k[t], v[t])
    got = W.kv4_block_values(block, hd)
    np.testing.assert_array_equal(got[0], W.kv4_round(k))
    np.testing.assert_array_equal(got[1], W.kv4_round(v))
