"""The numpy oracle of the 8-bit cache and the 4-bit products against values worked out by hand."""
import numpy as np
import pytest

from oracle import np_kv8


@pytest.mark.parametrize("top,e", [(0.0, -60), (127.0, 0), (127.00001, 1), (63.5, -1), (64.0, 0), (1.0, -6), (254.0, 1), (1e-30, -60), (np.inf, 127), (np.nan, 127)])
def test_exponents(top, e):
    assert np_kv8.exponent(np.array([0.0, -top])) == e


def test_a_block_that_grows():
    p = np_kv8.Part(2, 8)
    p.append(np.array([[127.0, -3.0]]))
    assert p.exps == [0] and p.codes.tolist() == [[127, -3]]
    p.append(np.array([[500.0, 2.0]]))  # units of 4: 127 / 4 = 31.75, -3 / 4 = -0.75, 125, 0.5 to even
    assert p.exps == [2] and p.codes.tolist() == [[32, -1], [125, 0]]
    p.append(np.zeros((7, 2)))
    assert p.exps == [2, -60] and len(p.codes) == 9
    p.append(np.array([[np.nan, 1.0]]))
    assert p.exps == [2, 127] and p.codes[8:].tolist() == [[0, 0], [0, 0]] and np.isnan(p.values()[8:]).all()


def test_attention_of_two_tokens():
    q, k, v = np.array([[1.0, 0.0]]), np.array([[np.log(3.0), 5.0], [0.0, 9.0]]), np.array([[4.0, 0.0], [0.0, 8.0]])
    out, p, bound, _ = np_kv8.attention(q, k, v, 1.0, [2])
    assert np.allclose(p, [[0.75, 0.25]], atol=1e-15) and np.allclose(out, [[3.0, 2.0]], atol=1e-14) and (bound < 0.02).all()
    assert (np_kv8.attention(q, k, v, 1.0, [0])[0] == 0).all()
    assert np.allclose(np_kv8.attention(q, k, v, 1.0, [1])[0], [[4.0, 0.0]])


def test_eviction_takes_equal_weights_by_slot():
    #       slot     0    1    2    3    4    5    6
    moves, w, p = np_kv8.evict([0.5, 0.1, 0.5, 0.9, 0.5, 0.0, 0.2], [0, 1, 2, 3, 4, 5, 6], 7, 4, 1)
    # 6 is recent, 3 is heaviest, of the equal ones 0 and 2 stay; 6 takes the place of 1
    assert moves == [(6, 1)] and w.tolist() == [0.5, 0.2, 0.5, 0.9] and p.tolist() == [0, 6, 2, 3]
    p = np_kv8.Part(1, 2)
    p.append(np.array([[100.0], [50.0], [3.0], [2.0], [200.0], [100.0]]))
    p.move([(5, 2)], 4)  # a unit of 2 comes into a block whose unit is 2^-5
    assert p.exps == [0, 1, 1] and p.codes[:, 0].tolist()[:4] == [100, 50, 50, 1]


def test_4_bit_products():
    y, bound = np_kv8.w4(np.array([[1.0, 2.0, 3.0]]), np.array([[0, 8, 15]]), np.array([[2.0, 0.5]]), np.array([[8, 7]]), 2)
    assert y.tolist() == [[1 * -8 * 2.0 + 0 + 3 * 8 * 0.5]] and 0 < bound[0, 0] < 1e-4
