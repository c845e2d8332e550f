"""The distillation oracle where the teacher's named probabilities sum above 1: finite differences (no GPU)."""
import numpy as np
import pytest

from oracle import head as H


@pytest.mark.parametrize("T", [0.7, 1.0, 3.0])
def test_gradient_against_differences_above_one(T):
    rng = np.random.default_rng(7)
    N, V, K = 4, 9, 3
    teacher, z = 2 * rng.normal(size=(N, V)), 2 * rng.normal(size=(N, V))
    ids = np.argsort(-teacher, 1)[:, :K]
    ids[2, 1] = ids[2, 0]                                 # named twice
    top = np.take_along_axis(teacher, ids, 1)
    lse = np.log(np.exp(top / T).sum(1) / np.array([1.5, 2.5, 1.05, 0.8]))       # the named probabilities' sums
    w = np.array([1.0, 0.5, 2.0, 1.0])
    loss, grad = H.distill(z, ids, top, T, lse, w)
    h = 1e-6
    for i in range(N):
        for j in range(V):
            d = np.zeros_like(z)
            d[i, j] = h
            num = (H.distill(z + d, ids, top, T, lse, w)[0].sum() - H.distill(z - d, ids, top, T, lse, w)[0].sum()) / (2 * h)
            assert abs(num - grad[i, j]) < 1e-6
    assert np.allclose(grad.sum(1), 0, atol=1e-12)
