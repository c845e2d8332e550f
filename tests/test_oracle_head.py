"""The output-head oracle against closed forms, brute force and finite differences (no GPU)."""
import math

import numpy as np
import pytest

from oracle import head as H


def test_e2m1_nearest_ties_and_saturation():
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    assert list(H.e2m1_nearest(np.array(mids))) == [0, 2, 2, 4, 4, 6, 6]
    assert list(H.e2m1_nearest(H.E2M1)) == list(range(8))
    assert list(H.e2m1_nearest(np.array([6.1, 1e30]))) == [7, 7]
    eps = 1e-9
    assert list(H.e2m1_nearest(np.array(mids) + eps)) == [1, 2, 3, 4, 5, 6, 7]
    assert list(H.e2m1_nearest(np.array(mids) - eps)) == [0, 1, 2, 3, 4, 5, 6]


def test_quantize_reproduces_representable_weights():
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 16, (5, 70))
    codes[:, 0::32] = 7                                   # every group of 32 reaches 6
    scales = 2.0 ** rng.integers(-3, 4, (5, 3))
    W = H.weights(codes, scales, 32)
    c, s = H.quantize(W, 32, lambda x: x.astype(np.float64), np.float64)
    assert np.allclose(s, scales, rtol=1e-7)
    assert np.array_equal(H.weights(c, scales, 32), W)
    packed = H.pack(c)
    assert packed.shape == (5, 48) and (packed[:, 35:] == 0).all()
    assert packed[2, 3] == c[2, 6] | c[2, 7] << 4


def test_sample_kept_small_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.1, 0.3, 0.1]))
    order, kept = H.sample_kept(l)
    assert list(order) == [1, 3, 0, 2, 4]
    assert np.allclose(kept / kept.sum(), [0.1, 0.4, 0.1, 0.3, 0.1])
    assert list(H.sample_kept(l, k=3)[1] > 0) == [True, True, False, True, False]     # ties by index
    assert list(H.sample_kept(l, p=0.45)[1] > 0) == [False, True, False, True, False]
    assert list(H.sample_kept(l, p=0.0)[1] > 0) == [False, True, False, False, False]
    assert list(H.sample_kept(l, mp=0.5)[1] > 0) == [False, True, False, True, False]
    assert list(H.sample_kept(l, k=2, p=0.5)[1] > 0) == [False, True, False, False, False]   # 0.4 >= 0.5 * 0.7


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [0.7, 1.0, 3.0])
def test_distill_gradient_against_differences(tail, T):
    rng = np.random.default_rng(7)
    N, V, K = 4, 9, 3
    teacher, z = 2 * rng.normal(size=(N, V)), 2 * rng.normal(size=(N, V))
    ids = np.argsort(-teacher, 1)[:, :K]
    ids[1, 2] = -1
    ids[2, 1] = ids[2, 0]                                 # named twice
    top = np.take_along_axis(teacher, np.maximum(ids, 0), 1)
    if tail:
        top[2, :2] -= math.log(4.0) * T                   # keeps the named mass below 1
    lse = np.log(np.exp(teacher / T).sum(1)) if tail else None
    w = np.array([1.0, 0.5, 2.0, 0.0])
    loss, grad = H.distill(z, ids, top, T, lse, w)
    h = 1e-6
    for i in range(N):
        for j in range(V):
            d = np.zeros_like(z)
            d[i, j] = h
            num = (H.distill(z + d, ids, top, T, lse, w)[0].sum() - H.distill(z - d, ids, top, T, lse, w)[0].sum()) / (2 * h)
            assert abs(num - grad[i, j]) < 1e-7
    assert loss[3] == 0 and not grad[3].any()
    assert np.allclose(grad.sum(1), 0, atol=1e-12)


def test_distill_closed_forms():
    # student equal to the teacher: no loss, no gradient, with the rest as a class
    z = np.array([[0.3, -1.0, 2.0, 0.5]])
    lse = np.log(np.exp(z).sum(1))
    loss, grad = H.distill(z, np.array([[2, 3]]), z[:, [2, 3]], 1.0, lse)
    assert abs(loss[0]) < 1e-15 and np.abs(grad).max() < 1e-15
    # one named token, renormalized: cross entropy of that token
    loss, grad = H.distill(z, np.array([[1]]), np.array([[5.0]]))
    assert abs(loss[0] - (lse[0] + 1.0)) < 1e-12
    # every token named: plain KL
    t = np.array([[1.0, 0.0, -1.0, 2.0]])
    p, q = np.exp(t) / np.exp(t).sum(), np.exp(z) / np.exp(z).sum()
    loss, grad = H.distill(z, np.array([[0, 1, 2, 3]]), t)
    assert abs(loss[0] - (p * np.log(p / q)).sum()) < 1e-12 and np.allclose(grad, q - p)
