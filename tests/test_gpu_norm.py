"""The norm, its 8-bit output and its gradient against the binary64 oracle (oracle/step.py).

Tolerances.  A sum of n terms is at most 72 terms in one thread (33 in registers, n / 1024 beyond) and 6 + 16 joins:
relative error of the sum of squares 94 * 2^-24, of its root half of that, and a few roundings more: y within 60 * 2^-24 of
its size and half a step of its type.  Products and mixed-sign sums: the same number of roundings of the sum of
magnitudes."""
import numpy as np
import pytest

from oracle import step as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def half_step(prec):
    return torch.finfo(DT[prec]).eps / 2


def tiny(prec):
    """Half the spacing of the type's subnormal numbers."""
    return torch.finfo(DT[prec]).smallest_normal * torch.finfo(DT[prec]).eps / 2


def rand(seed, *shape, size=1.0, prec="fp32"):
    rng = np.random.default_rng([seed, *shape])
    return torch.from_numpy(rng.normal(size=shape) * size).to(DT[prec]).cuda()


def pitched(t, more):
    """t in rows of a larger pitch, not aligned to 16 bytes."""
    big = torch.full((t.shape[0], t.shape[1] + more), float("nan"), dtype=t.dtype, device="cuda")
    v = big[:, 1:1 + t.shape[1]]
    v.copy_(t)
    return v


def host(t):
    return t.double().cpu().numpy()


SIZES = [(1, 1), (1, 7), (3, 8), (2, 255), (5, 256), (4, 1003), (1, 8192), (2, 16384), (1, 33000), (3, 70001), (600, 130),
         (513, 2048), (530, 4100), (515, 8200)]


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("residual,wprec", [(True, "same"), (False, "fp32"), (True, None), (False, "other")])
def test_norm(lrc, prec, rows, n, residual, wprec):
    wprec = {"same": prec, "other": "fp16" if prec == "bf16" else "bf16"}.get(wprec, wprec)
    x = rand(1, rows, n, prec=prec)
    res = rand(2, rows, n, size=3.0, prec=prec) if residual else None
    w = None if wprec is None else (1.0 + rand(3, n, size=0.2)).to(DT[wprec])
    if rows <= 4:
        x, res = pitched(x, 5), pitched(res, 3) if residual else None
    y, h, rstd = lrc.rms_norm(x, w, residual=res, eps=1e-5, stats=True)
    want_h = (x.double() + res.double()).to(DT[prec]) if residual else x
    assert torch.equal(h, want_h)
    yw, rw = O.rms_norm(host(h), None if w is None else host(w), 1e-5)
    assert np.all(np.abs(host(rstd) - rw) <= 60 * U * rw)
    assert np.all(np.abs(host(y) - yw) <= (half_step(prec) + 60 * U) * np.abs(yw) + tiny(prec))
    # the residual's place takes the sum
    if residual:
        y2, h2 = lrc.rms_norm(x, w, residual=res, eps=1e-5, sum=res)
        assert h2 is res and torch.equal(res, want_h) and torch.equal(y2, y)


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,n", SIZES)
def test_norm_in_8_bits(lrc, prec, rows, n):
    x, res = rand(4, rows, n, prec=prec), rand(5, rows, n, size=2.0, prec=prec)
    x[0] *= 2.0 ** -6
    w = 1.0 + rand(6, n, size=0.2)
    codes, scales, h = lrc.rms_norm_e4m3(x, w, residual=res)
    assert torch.equal(h, (x.double() + res.double()).to(DT[prec]))
    yw, _ = O.rms_norm(host(h), host(w))
    tw = np.abs(yw).max(1) / 448.0
    t = host(scales)
    assert np.all(np.abs(t - tw) <= 62 * U * tw)
    q = yw / t[:, None]
    step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -7))) - 3), 2.0 ** -9)
    got = host(codes.float())
    assert np.all(np.abs(got - q) <= step / 2 + 62 * U * np.abs(q))
    # away from the middles of two values the code is the nearest one
    far = np.abs(O.e4m3_nearest(q * (1 + 1e-4)) - O.e4m3_nearest(q * (1 - 1e-4))) == 0
    assert far.mean() > 0.9 or n < 64
    assert np.array_equal(got[far], O.e4m3_nearest(q)[far])


def test_rows_of_zeros_and_not_finite(lrc):
    n = 1000
    for prec in DT:
        x = rand(7, 6, n, prec=prec)
        x[0] = 0
        x[1, 3] = float("nan")
        x[2, n - 1] = float("inf")
        x[3] = 0
        x[3, 5] = 2.0 ** -14
        codes, scales, _ = lrc.rms_norm_e4m3(x, None)
        got, t = host(codes.float()), host(scales)
        assert np.all(got[0] == 0) and t[0] == 0
        assert np.isnan(got[1]).all() and np.isnan(t[1]) and np.isnan(got[2]).all() and np.isnan(t[2])
        assert got[3, 5] == 448 and np.count_nonzero(got[3]) == 1
        assert np.isfinite(got[4:]).all() and np.isfinite(t[4:]).all()
        y, _ = lrc.rms_norm(x, None)
        assert host(y)[0].any() == False and np.isnan(host(y)[1]).all()      # noqa: E712
        assert np.isfinite(host(y)[3:]).all()
    # magnitudes whose scale is subnormal, or none at all
    x = torch.full((3, 64), 2.0 ** -60, device="cuda")
    x[0, 0], x[1, 0] = 2.0 ** -55, 2.0 ** -62
    w = torch.full((64,), 2.0 ** -80, device="cuda")
    codes, scales, _ = lrc.rms_norm_e4m3(x, w, eps=1e-6)
    v = host(codes.float()) * host(scales)[:, None]
    want, _ = O.rms_norm(host(x), host(w))
    assert np.all(np.abs(host(codes.float())) <= 448) and np.all(np.abs(v - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -139)


def test_no_rows(lrc):
    for prec in DT:
        x = torch.empty(0, 40, dtype=DT[prec], device="cuda")
        y, h, r = lrc.rms_norm(x, None, residual=x, stats=True)
        assert y.shape == (0, 40) and r.shape == (0,)
        w = torch.ones(40, device="cuda")
        dx, dw = lrc.rms_norm_backward(x, h, w, r)
        assert dx.shape == (0, 40) and not dw.any()


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,n", SIZES + [(1030, 600), (2100, 33)])
@pytest.mark.parametrize("dsum,wprec", [(True, "same"), (False, "fp32"), (True, None)])
def test_gradient(lrc, prec, rows, n, dsum, wprec):
    wprec = prec if wprec == "same" else wprec
    h, dy = rand(8, rows, n, prec=prec), rand(9, rows, n, prec=prec)
    ds = rand(10, rows, n, prec=prec) if dsum else None
    w = None if wprec is None else (1.0 + rand(11, n, size=0.2)).to(DT[wprec])
    if rows <= 4:
        h, dy, ds = pitched(h, 4), pitched(dy, 7), pitched(ds, 2) if dsum else None
    _, _, rstd = lrc.rms_norm(h, w, stats=True)
    dx, dw = lrc.rms_norm_backward(dy, h, w, rstd, dsum=ds)
    H, D, W = host(h), host(dy), 1.0 if w is None else host(w)
    dxw, dww = O.rms_norm_backward(D, H, None if w is None else W, dsum=host(ds) if dsum else None)
    r = 1.0 / np.sqrt((H * H).mean(1, keepdims=True) + 1e-6)
    size = r * np.abs(D * W) + np.abs(H) * r ** 3 * np.abs(D * W * H).mean(1, keepdims=True)
    assert np.all(np.abs(host(dx) - dxw) <= half_step(prec) * np.abs(dxw) + 250 * U * size + 2 * U * np.abs(dxw) + tiny(prec))
    if w is None:
        assert dw is None
    else:
        # at most rows / 256 (one group of rows) + groups / 16 + 16 additions
        depth = rows / 256 + 4096 / 16 + 80
        bound = half_step(wprec) * np.abs(dww) + depth * U * np.abs(D * H * r).sum(0) + tiny(wprec)
        assert np.all(np.abs(host(dw) - dww) <= bound)
    again = lrc.rms_norm_backward(dy, h, w, rstd, dsum=ds)
    assert torch.equal(again[0], dx) and (w is None or torch.equal(again[1], dw))
    # in the place of dy
    mine = dy.clone()
    assert torch.equal(lrc.rms_norm_backward(mine, h, w, rstd, dsum=ds, dx=mine)[0], dx)


def test_gradient_against_differences(lrc):
    rows, n = 6, 300
    h, dy, w = rand(12, rows, n), rand(13, rows, n), 1.0 + rand(14, n, size=0.3)
    _, _, rstd = lrc.rms_norm(h, w, stats=True)
    dx, dw = lrc.rms_norm_backward(dy, h, w, rstd)
    f = lambda H, W: (O.rms_norm(H, W)[0] * host(dy)).sum()  # noqa: E731
    rng = np.random.default_rng(15)
    for _ in range(5):
        v, s = rng.normal(size=(rows, n)), rng.normal(size=n)
        e = 1e-5
        num = (f(host(h) + e * v, host(w)) - f(host(h) - e * v, host(w))) / (2 * e)
        # differences: e^2 times third derivatives; the gradient: binary32
        assert abs(num - (host(dx) * v).sum()) <= 1e-5 * np.abs(host(dx) * v).sum()
        num = (f(host(h), host(w) + e * s) - f(host(h), host(w) - e * s)) / (2 * e)
        assert abs(num - (host(dw) * s).sum()) <= 1e-5 * np.abs(host(dw) * s).sum()
