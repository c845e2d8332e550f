"""Adapters and their gradient against the binary64 oracle (oracle/step.py).

Tolerances count roundings.  A sum of L products in binary32 is within L * 2^-24 of the sum of magnitudes, whatever its
order; hidden values enter the second product as pairs of 16-bit values, within 2^-16 (bfloat16: 2^-9 of 2^-8) or 2^-20
(binary16: 2^-12 of 2^-11, of the largest of the row at least 2^-24) of themselves, and the result is rounded once."""
import numpy as np
import pytest

from oracle import step as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24
PAIR = {"fp32": 0.0, "fp16": 2.0 ** -20, "bf16": 2.0 ** -16}


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def half_step(prec):
    return torch.finfo(DT[prec]).eps / 2


def tiny(prec):
    return torch.finfo(DT[prec]).smallest_normal * torch.finfo(DT[prec]).eps / 2


def host(t):
    return None if t is None else t.double().cpu().numpy()


def rand(rng, *shape, size=1.0, prec="fp32"):
    return torch.from_numpy(rng.normal(size=shape) * size).to(DT[prec]).cuda()


def pitched(t, more):
    big = torch.full((t.shape[0], t.shape[1] + more), float("nan"), dtype=t.dtype, device="cuda")
    v = big[:, 1:1 + t.shape[1]]
    v.copy_(t)
    return v


def ids_of(rng, rows, count, kind):
    if kind == "none":
        ids = np.full(rows, -1)
    elif kind == "one":
        ids = np.full(rows, count - 1)
    elif kind == "runs":
        ids = np.sort(rng.integers(-1, count, rows))
    else:
        ids = rng.integers(-1, count + 1, rows)          # -1 and count name none
    return torch.from_numpy(ids.astype(np.int64)).cuda()


SIZES = [(1, 1, 1, 1, 1, "one"), (1, 512, 256, 8, 4, "any"), (5, 33, 65, 3, 2, "any"), (48, 130, 600, 16, 7, "any"),
         (64, 257, 1025, 200, 9, "any"), (64, 40, 64, 256, 2, "runs"), (65, 129, 257, 17, 3, "any"), (66, 1, 1, 1, 1, "one"),
         (200, 300, 130, 64, 5, "runs"), (100, 64, 520, 256, 3, "any"), (130, 260, 140, 130, 70, "any"), (700, 96, 160, 128, 2, "runs"),
         (1500, 70, 90, 5, 1, "one"), (1100, 50, 70, 40, 3, "any"), (300, 40, 50, 8, 400, "any"), (150, 66, 34, 12, 3, "none"),
         (513, 140, 300, 32, 1, "one"), (1030, 128, 256, 16, 2, "runs")]


def problem(seed, rows, m, n, k, count, kind, prec):
    rng = np.random.default_rng([seed, rows, m, n, k])
    return dict(X=rand(rng, rows, n, prec=prec), A=rand(rng, count, k, n, size=n ** -0.5, prec=prec),
                B=rand(rng, count, m, k, size=k ** -0.5, prec=prec), ids=ids_of(rng, rows, count, kind),
                scale=torch.from_numpy(rng.uniform(0.5, 2.0, count).astype(np.float32)).cuda(),
                base=rand(rng, rows, m, prec=prec), dY=rand(rng, rows, m, prec=prec), dbase=rand(rng, rows, n, prec=prec))


def bounds(q, prec, scale=True):
    """Tolerances of Y, hidden, dX, dA and dB, and their oracle values."""
    X, A, B, ids = host(q["X"]), host(q["A"]), host(q["B"]), q["ids"].cpu().numpy()
    c = host(q["scale"]) if scale else np.ones(len(A))
    dY, base, dbase = host(q["dY"]), host(q["base"]), host(q["dbase"])
    rows, n = X.shape
    m, k = B.shape[1:]
    Y, H = O.adapters(X, A, B, ids, c, base)
    dX, dA, dB = O.adapters_backward(dY, X, A, B, ids, c, dbase)
    eps, pair = half_step(prec), PAIR[prec]
    bY, bH, bX = eps * np.abs(Y) + 2 * U * np.abs(base), np.zeros(H.shape), eps * np.abs(dX) + 2 * U * np.abs(dbase)
    bA, bB = eps * np.abs(dA), eps * np.abs(dB)
    floor16 = 2.0 ** -24 if prec == "fp16" else 0.0
    for i, a in enumerate(ids):
        if not 0 <= a < len(A):
            continue
        size = np.abs(A[a]) @ np.abs(X[i])
        bH[i] = (n + 8) * U * size
        big = floor16 * np.abs(H[i]).max()
        bY[i] += c[a] * np.abs(B[a]) @ (bH[i] + (pair + (k + 4) * U) * size + big)
        dsize = c[a] * np.abs(dY[i]) @ np.abs(B[a])
        derr = (m + 8) * U * dsize
        big = floor16 * dsize.max()
        bX[i] += (derr + (pair + (k + 4) * U) * dsize + big) @ np.abs(A[a])
        bA[a] += np.outer(derr + (pair + (rows + 8) * U) * dsize, np.abs(X[i]))
        bB[a] += c[a] * np.outer(np.abs(dY[i]), bH[i] + (pair + (rows + 8) * U) * size)
    if prec == "fp16":          # pairs over rows: 2^-24 of the largest value of a rank in up to 512 rows
        for a in range(len(A)):
            r = np.flatnonzero(ids == a)
            if len(r):
                dh = np.abs(c[a] * dY[r] @ B[a]).max(0)
                bA[a] += 2.0 ** -24 * np.outer(dh, np.abs(X[r]).sum(0))
                bB[a] += 2.0 ** -24 * c[a] * np.outer(np.abs(dY[r]).sum(0), np.abs(H[r]).max(0))
    return (Y, bY), (H, bH), (dX, bX), (dA, bA), (dB, bB)


def near(got, pair, prec, what):
    want, bound = pair
    off = np.abs(host(got) - want)
    assert np.all(off <= bound + tiny(prec)), (what, float((off - bound).max()))


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_adapters(lrc, prec, size):
    q = problem(1, *size, prec)
    (Y, H, dX, dA, dB) = bounds(q, prec)
    got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], scale=q["scale"], base=q["base"], hidden=True)
    near(hidden, H, "fp32", "hidden")
    near(got, Y, prec, "Y")
    assert torch.equal(got, lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], scale=q["scale"], base=q["base"]))
    none = (q["ids"] < 0) | (q["ids"] >= size[4])
    assert torch.equal(got[none], q["base"][none])
    # in the place of the base, rows of other pitches
    mine = pitched(q["base"], 3)
    lrc.adapter_apply(pitched(q["X"], 5), q["A"], q["B"], q["ids"], scale=q["scale"], base=mine, Y=mine)
    assert torch.equal(mine, got)
    grads = lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden, scale=q["scale"], base=q["dbase"])
    for g, w, what in zip(grads, (dX, dA, dB), ("dX", "dA", "dB")):
        near(g, w, prec, what)
    assert torch.equal(grads[0][none], q["dbase"][none])
    mine = pitched(q["dbase"], 1)
    again = lrc.adapter_backward(pitched(q["dY"], 2), pitched(q["X"], 4), q["A"], q["B"], q["ids"], hidden, scale=q["scale"],
                                 base=mine, dX=mine)
    for g, w in zip(again, grads):
        assert torch.equal(g, w)


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows", [3, 90])
def test_without_scale_and_base(lrc, prec, rows):
    q = problem(2, rows, 70, 90, 12, 4, "any", prec)
    q["base"].zero_(), q["dbase"].zero_()
    (Y, H, dX, dA, dB) = bounds(q, prec, scale=False)
    got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], hidden=True)
    near(got, Y, prec, "Y")
    for g, w, what in zip(lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden), (dX, dA, dB), ("dX", "dA", "dB")):
        near(g, w, prec, what)


@pytest.mark.parametrize("rows", [40, 600])
def test_what_is_not_finite_stays_in_its_row(lrc, rows):
    """NaN and infinities of rows without an adapter, and of one adapter's row, reach nothing else."""
    for prec in DT:
        q = problem(3, rows, 100, 140, 16, 3, "any", prec)
        none = torch.nonzero(q["ids"] < 0)[:, 0]
        q["X"][none] = float("nan")
        q["dY"][none[0]] = float("inf")
        bad = int(torch.nonzero(q["ids"] == 1)[0])
        q["X"][bad, 7] = float("nan")
        got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], base=q["base"], hidden=True)
        fine = torch.ones(rows, dtype=torch.bool, device="cuda")
        fine[bad] = False
        assert torch.isfinite(got[fine]).all() and torch.isnan(got[bad]).all()
        assert torch.equal(got[none], q["base"][none])
        dX, dA, dB = lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden)
        assert torch.isfinite(dX).all()
        assert torch.isfinite(dA[[0, 2]]).all() and torch.isfinite(dB[[0, 2]]).all()
        assert torch.isnan(dA[1, :, 7]).all() and torch.isfinite(dA[1, :, 8:]).all() and torch.isnan(dB[1]).all()


@pytest.mark.parametrize("rows", [20, 200])
@pytest.mark.parametrize("up,down", [(2.0 ** 10, 2.0 ** -12), (2.0 ** -11, 2.0 ** 6)])
def test_hidden_values_out_of_binary16_range(lrc, rows, up, down):
    """Hidden values of 1e6 and of 1e-6 in binary16 calls: pairs carry the range of their row."""
    q = problem(4, rows, 60, 400, 24, 2, "any", "fp16")
    q["X"] *= up
    q["A"] *= up / 8
    q["B"] *= down
    q["base"].zero_(), q["dbase"].zero_()
    q["dY"] *= 2.0 ** -3
    Y, H, dX, dA, dB = bounds(q, "fp16")
    got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], scale=q["scale"], hidden=True)
    assert np.isfinite(Y[0]).all() and np.abs(Y[0]).max() < 6e4
    near(got, Y, "fp16", "Y")
    grads = lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden, scale=q["scale"])
    for g, w, what in zip(grads, (dX, dA, dB), ("dX", "dA", "dB")):
        keep = np.abs(w[0]) < 6.5e4                       # larger ones are infinite in binary16
        off = np.abs(host(g) - w[0])
        assert np.all(off[keep] <= (w[1] + tiny("fp16"))[keep]), what


def test_many_adapters(lrc):
    """Five digits of keys; most adapters without rows."""
    rng = np.random.default_rng(5)
    count, rows, m, n, k = 70000, 500, 9, 11, 2
    ids = rng.choice([0, 1, 15, 16, 255, 256, 4095, 65535, 65536, 69999, 70000], rows)
    q = problem(6, rows, m, n, k, count, "any", "bf16")
    q["ids"] = torch.from_numpy(ids).cuda()
    Y, H, dX, dA, dB = bounds(q, "bf16")
    got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], scale=q["scale"], base=q["base"], hidden=True)
    near(got, Y, "bf16", "Y")
    grads = lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden, scale=q["scale"], base=q["dbase"])
    for g, w, what in zip(grads, (dX, dA, dB), ("dX", "dA", "dB")):
        near(g, w, "bf16", what)


def test_no_rows(lrc):
    q = problem(7, 4, 30, 20, 5, 3, "any", "bf16")
    e = q["X"][:0]
    Y, H = lrc.adapter_apply(e, q["A"], q["B"], q["ids"][:0], hidden=True)
    assert Y.shape == (0, 30) and H.shape == (0, 5)
    dX, dA, dB = lrc.adapter_backward(q["dY"][:0], e, q["A"], q["B"], q["ids"][:0], H)
    assert dX.shape == (0, 20) and not dA.any() and not dB.any()


def test_gradient_against_differences(lrc):
    q = problem(8, 90, 40, 50, 6, 3, "any", "fp32")
    got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], scale=q["scale"], hidden=True)
    dX, dA, dB = map(host, lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden, scale=q["scale"]))
    X, A, B, ids, c, dY = (host(q[x]) for x in ("X", "A", "B", "ids", "scale", "dY"))
    f = lambda X, A, B: (O.adapters(X, A, B, ids.astype(int), c)[0] * dY).sum()  # noqa: E731
    rng = np.random.default_rng(9)
    for _ in range(4):
        vX, vA, vB = rng.normal(size=X.shape), rng.normal(size=A.shape), rng.normal(size=B.shape)
        e = 1e-5
        num = (f(X + e * vX, A + e * vA, B + e * vB) - f(X - e * vX, A - e * vA, B - e * vB)) / (2 * e)
        size = np.abs(dX * vX).sum() + np.abs(dA * vA).sum() + np.abs(dB * vB).sum()
        assert abs(num - ((dX * vX).sum() + (dA * vA).sum() + (dB * vB).sum())) <= 1e-5 * size
