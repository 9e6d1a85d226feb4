"""Pins of the 8-bit cache's oracle: closed forms that need no other implementation."""
import numpy as np
import pytest

from oracle import cache_oracle as C


@pytest.mark.parametrize("top,scale", [(127.0, 1.0), (127.00001, 2.0), (63.5, 0.5), (1.0, 2.0 ** -6), (0.0, 2.0 ** -60), (1e-30, 2.0 ** -60),
                                       (254.0, 2.0), (3e38, 2.0 ** 60)])
def test_scale_is_the_smallest_power_of_two(top, scale):
    assert C.block_scale(np.array([0.0, -top])) == scale


def test_codes_round_half_to_even():
    assert C.codes(np.array([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 127.4]), 1.0).tolist() == [0, 2, 2, 0, -2, 126, 127]


def test_a_block_that_grows_moves_its_rows_to_the_larger_scale():
    h = C.Head(2)
    h.store(np.array([[1.0, 0.25]]), np.zeros((1, 2)))
    assert h.ks == [2.0 ** -6] and h.k.tolist() == [[1.0, 0.25]]
    h.store(np.array([[100.0, 0.0]]), np.zeros((1, 2)))
    assert h.ks == [1.0] and h.k.tolist() == [[1.0, 0.0], [100.0, 0.0]] and h.ids == [0, 1]
    h.store(np.ones((63, 2)), np.zeros((63, 2)), pos=10)
    assert len(h.ks) == 2 and h.ks[1] == 2.0 ** -6 and h.ids[2] == 10 and len(h) == 65


def test_eviction_keeps_recent_rows_then_weights_then_the_earlier_of_equals():
    h = C.Head(1)
    h.store(np.arange(6.0)[:, None], np.zeros((6, 1)))
    h.weights = [0.5, 0.0, 2.0, 0.5, 0.0, float("nan")]
    h.evict(4, 1, 6)                       # row 5 is recent; then 2, 0, 3
    assert h.ids == [0, 5, 2, 3] and h.k[:, 0].tolist() == [0.0, 5.0, 2.0, 3.0]
    h.evict(1, 0, 6)
    assert h.ids == [2]


def test_attention_of_equal_keys_is_the_mean():
    h = C.Head(4)
    v = np.arange(12.0).reshape(3, 4)
    h.store(np.ones((3, 4)), v)
    out, p, _, _ = h.attend(np.ones((2, 4)))
    assert np.allclose(out, v.mean(0)) and np.allclose(p, 1 / 3)


def test_packed_prompts_do_not_see_each_other_and_weights_sum_to_the_queries():
    g = np.random.default_rng(0)
    q, k, v = g.normal(size=(7, 4, 8)), g.normal(size=(7, 2, 8)), g.normal(size=(7, 2, 8))
    out, lse, _, _ = C.packed_attend(q, k, v, [3, 0, 4])
    alone, lse1, _, _ = C.packed_attend(q[3:], k[3:], v[3:], [4])
    assert np.allclose(out[3:], alone) and np.allclose(lse[:, 3:], lse1) and np.allclose(out[0], v[0].repeat(2, 0))
    w = C.packed_weights(q, k, lse, [3, 0, 4])
    assert [x.shape for x in w] == [(2, 3), (2, 0), (2, 4)]
    assert np.allclose(w[0].sum(), 3 * 4) and np.allclose(w[2].sum(), 4 * 4)
    assert np.allclose(C.packed_weights(q, k, lse, [3, 0, 4], window=1)[2].sum(1), 2)
