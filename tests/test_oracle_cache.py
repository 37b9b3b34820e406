"""Pins of the oracle's 4-bit rows, key weights and eviction."""
import numpy as np
import pytest


def rand(shape, seed):
    return np.random.default_rng(seed).standard_normal(shape)


def test_row_weights_are_the_rows_of_the_full_matrix(oracle):
    q, k = rand((9, 4), 1), rand((9, 4), 2)
    A, _, rem = oracle.weights(q, k)
    for j in range(9):
        a, left = oracle.row_weights(q[j], k[:j])
        assert np.abs(a - A[j, :j]).max(initial=0.0) < 1e-15 and abs(left - rem[j]) < 1e-15


def test_key_weight_sums_the_columns(oracle):
    q, k = rand((2, 4, 7, 4), 3), rand((2, 2, 7, 4), 4)
    got = oracle.key_weight(q, k)
    for b in range(2):
        for g in range(2):
            want = sum(oracle.weights(q[b, h], k[b, g])[0].sum(0) for h in (2 * g, 2 * g + 1))
            assert np.abs(got[b, g] - want).max() < 1e-14
    # a window at the end, and entries of different lengths: those rows alone
    window = oracle.key_weight(q[:, :, 4:], k)
    padded = oracle.key_weight(q, k, lens=[7, 3], qlens=[7, 3])
    for b in range(2):
        for h in range(4):
            A = oracle.weights(q[b, h], k[b, h // 2])[0]
            window[b, h // 2] -= A[4:].sum(0)
            padded[b, h // 2] -= A[:(7, 3)[b]].sum(0)
    assert np.abs(window).max() < 1e-14 and np.abs(padded).max() < 1e-14


@pytest.mark.parametrize("top,byte", [(0.0, 7), (1e-40, 7), (7.0, 127), (7.001, 128), (3.5, 126), (6.0, 127), (3.4e38, 253)])
def test_scale_of_a_block(oracle, top, byte):
    x = np.zeros(32)
    x[5] = -top
    assert int(oracle.kv4(x)[1][0]) == byte


def test_rounding_of_a_block(oracle):
    x = np.zeros(32)
    x[:16] = [7.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, -0.25, -0.75, -3.5, -6.9, 0.0, 4.0]
    codes, scales = oracle.kv4(x)
    want = [6.0, 0.0, 0.5, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 0.0, -1.0, -4.0, -6.0, 0.0, 4.0]
    assert oracle.kv4_values(codes, scales)[:16].tolist() == want


def test_rounding_is_within_half_a_step(oracle):
    x = rand((50, 96), 5) * np.exp(3 * rand((50, 1), 6))
    codes, scales = oracle.kv4(x)
    y, unit = oracle.kv4_values(codes, scales), np.repeat(2.0 ** (scales - 127.0), 32, axis=-1)
    step = np.where(np.abs(x) <= 2 * unit, 0.25, np.where(np.abs(x) <= 4 * unit, 0.5, 1.0)) * unit
    assert (np.abs(x - y) <= step).all()
    again = oracle.kv4(y)
    assert np.array_equal(oracle.kv4_values(*again), y)


def test_eviction(oracle):
    s = [5.0, 1.0, 1.0, 9.0, 0.0, 2.0]
    assert oracle.evict(s, 6, 4, 1) == [0, 1, 3, 5]            # of the two ones the first
    assert oracle.evict(s, 6, 4, 4) == [2, 3, 4, 5]
    assert oracle.evict(s, 4, 4, 0) == [0, 1, 2, 3] and oracle.evict(s, 0, 4, 0) == []
