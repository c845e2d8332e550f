"""The oracle of the norm, the adapters, e4m3 and the verification against definitions, differences and counts (no GPU)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import step as O  # noqa: E402


def test_e4m3_is_torchs_nearest():
    assert np.array_equal(O.E4M3, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    rng = np.random.default_rng(1)
    mids = (O.E4M3[1:] + O.E4M3[:-1]) / 2
    a = np.concatenate([mids, -mids, O.E4M3, rng.normal(size=4000) * 10.0 ** rng.uniform(-4, 2, 4000)])
    a = a[np.abs(a) <= 448].astype(np.float32)
    want = torch.from_numpy(a).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_nearest(a), want)
    assert np.array_equal(O.e4m3_nearest([1e9, -500.0]), [448.0, -448.0])


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(2)
    h, w, dy, ds = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    y, rstd = O.rms_norm(h, w)
    assert np.allclose(y, h / np.sqrt((h ** 2).sum(1, keepdims=True) / 7 + 1e-6) * w, rtol=1e-14) and rstd.shape == (3,)
    dx, dw = O.rms_norm_backward(dy, h, w, dsum=ds)
    f = lambda h, w: (O.rms_norm(h, w)[0] * dy).sum() + (h * ds).sum()  # noqa: E731
    e = 1e-6
    for _ in range(5):
        vh, vw = rng.normal(size=h.shape), rng.normal(size=7)
        num = (f(h + e * vh, w + e * vw) - f(h - e * vh, w - e * vw)) / (2 * e)
        assert abs(num - ((dx * vh).sum() + (dw * vw).sum())) < 1e-7


def test_adapter_gradients_against_differences():
    rng = np.random.default_rng(3)
    X, A, B, dY, c = (rng.normal(size=s) for s in ((6, 5), (3, 2, 5), (3, 4, 2), (6, 4), (3,)))
    ids = np.array([0, 2, -1, 2, 3, 0])
    base, dbase = rng.normal(size=(6, 4)), rng.normal(size=(6, 5))
    Y, H = O.adapters(X, A, B, ids, c, base)
    assert np.array_equal(Y[[2, 4]], base[[2, 4]]) and not H[[2, 4]].any()
    assert np.allclose(Y[1], base[1] + c[2] * B[2] @ (A[2] @ X[1]), rtol=1e-14)
    dX, dA, dB = O.adapters_backward(dY, X, A, B, ids, c, dbase)
    assert not dA[1].any() and not dB[1].any() and np.array_equal(dX[2], dbase[2])
    f = lambda X, A, B: (O.adapters(X, A, B, ids, c)[0] * dY).sum() + (X * dbase).sum()  # noqa: E731
    e = 1e-6
    for _ in range(5):
        v = [rng.normal(size=t.shape) for t in (X, A, B)]
        num = (f(X + e * v[0], A + e * v[1], B + e * v[2]) - f(X - e * v[0], A - e * v[1], B - e * v[2])) / (2 * e)
        assert abs(num - sum((g * t).sum() for g, t in zip((dX, dA, dB), v))) < 1e-6


def test_verification_by_hand():
    P = np.array([[4, 4, 0], [1, 3, 0], [0, 0, 8]])
    assert O.verify(P, [0, 1], np.array([0.4, 0.7, 0.5])) == ([0, 1, 2], 2)            # certain drafts: u < p
    assert O.verify(P, [0, 1], np.array([0.6, 0.7, 0.5])) == ([1, -1, -1], 0)          # what is left of (1/2, 1/2) is token 1
    assert O.verify(P, [0, 3], np.array([0.4, 0.0, 0.2])) == ([0, 0, -1], 1)           # no token: drawn from P
    assert O.verify(P, [2, 0], np.array([0.0, 0.0, 0.1])) == ([0, -1, -1], 0)          # weight 0 is never accepted
    Q = np.array([[1, 7, 0], [1, 3, 0]])
    assert O.verify(P, [1, 0], np.array([0.58, 0.99, 0.9]), Q)[0] == [0, -1, -1]       # 0.58 * 7/8 > 1/2, left: token 0
    assert O.verify(P, [1, 0], np.array([0.56, 0.99, 0.9]), Q) == ([1, 0, 2], 2)       # equal distributions accept
    assert O.verify(np.zeros((1, 3)), [], np.array([0.3])) == ([-1], 0)


@pytest.mark.parametrize("certain", [False, True])
def test_verified_tokens_follow_the_target(certain):
    """The first token's law is the target's: integrated over u on a grid of midpoints, with weights whose products with
    the grid are whole."""
    P, Q = np.array([[1, 4, 3, 0], [1, 1, 1, 1]]), np.array([[4, 2, 1, 1]])
    G = 64
    mass = np.zeros(4)
    for draft in range(4):
        share = float(Q[0, draft]) / 8 if not certain else float(draft == 1)
        if share == 0:
            continue
        for i in range(G):
            for j in range(G):
                out, _ = O.verify(P, [draft], np.array([(i + 0.5) / G, (j + 0.5) / G]), None if certain else Q)
                mass[out[0]] += share / G ** 2
    # acceptance exact on the grid (G times every ratio is whole); the drawn token's share of the rest within 4 steps
    assert np.abs(mass - P[0] / 8).max() <= 4.0 / G
