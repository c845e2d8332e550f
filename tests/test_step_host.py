"""Refusals of the norm, adapter and verification calls and of 8-bit activations, C ABI and binding (no GPU needed): every
check runs before any device call."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_12969_amd import lrc  # noqa: E402

A = [0x1000000 * (i + 1) for i in range(14)]
INVALID, OVERFLOW, NODEV = -1, -2, -5
E4M3 = 4


def L():
    return lrc.lib()


def nodev():
    return not torch.cuda.is_available()


def norm(x=A[0], ldx=100, res=A[1], ldr=100, rows=4, n=100, prec=1, w=A[2], wprec=1, eps=1e-6, sum=A[3], lds=100, y=A[4], ldy=100,
         yprec=1, scales=None, rstd=A[6]):
    return L().lrc_rms_norm(x, ldx, res, ldr, rows, n, prec, w, wprec, eps, sum, lds, y, ldy, yprec, scales, rstd)


def test_norm_refusals():
    for kw in (dict(x=None), dict(y=None), dict(rows=-1), dict(n=0), dict(prec=0, yprec=0), dict(prec=E4M3), dict(wprec=E4M3), dict(yprec=2),
               dict(yprec=E4M3), dict(scales=A[5]), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e39),
               dict(ldx=99), dict(ldr=99), dict(lds=99), dict(ldy=99), dict(ldx=0),
               dict(y=A[0]), dict(y=A[1]), dict(y=A[2] + 4), dict(y=A[3] + 8), dict(sum=A[0] + 2), dict(sum=A[1] + 2),
               dict(sum=A[0], lds=101), dict(sum=A[1], lds=104), dict(sum=A[2]), dict(rstd=A[0]), dict(rstd=A[3]), dict(rstd=A[4]),
               dict(yprec=E4M3, scales=A[6]), dict(yprec=E4M3, scales=A[4])):
        assert norm(**kw) == INVALID, kw
    assert norm(ldx=2 ** 62) == OVERFLOW and norm(rows=2 ** 61) == OVERFLOW
    assert norm(rows=0, x=None, y=None, res=None, sum=None) == 0
    if nodev():
        for kw in (dict(), dict(sum=A[0]), dict(sum=A[1]), dict(sum=None), dict(res=None, sum=None), dict(rstd=None), dict(w=None),
                   dict(eps=0.0), dict(yprec=E4M3, scales=A[5])):
            assert norm(**kw) == NODEV, kw


def norm_back(dy=A[0], lddy=100, h=A[1], ldh=100, rstd=A[2], rows=4, n=100, prec=1, w=A[3], wprec=1, ds=A[4], ldd=100, dx=A[5],
              ldx=100, dw=A[6]):
    return L().lrc_rms_norm_backward(dy, lddy, h, ldh, rstd, rows, n, prec, w, wprec, ds, ldd, dx, ldx, dw)


def test_norm_gradient_refusals():
    for kw in (dict(dy=None), dict(h=None), dict(rstd=None), dict(dx=None), dict(rows=-1), dict(n=0), dict(prec=E4M3), dict(wprec=E4M3),
               dict(w=None, wprec=9), dict(lddy=99), dict(ldh=99), dict(ldd=99), dict(ldx=99), dict(dx=A[1]), dict(dx=A[0] + 2),
               dict(dx=A[4] + 2), dict(dx=A[0], ldx=101), dict(dx=A[2]), dict(dx=A[3]), dict(dw=A[0]), dict(dw=A[3]), dict(dw=A[5]),
               dict(dw=A[2])):
        assert norm_back(**kw) == INVALID, kw
    assert norm_back(lddy=2 ** 62) == OVERFLOW and norm_back(rows=1, n=2 ** 58, lddy=2 ** 58, ldh=2 ** 58, ldd=2 ** 58,
                                                            ldx=2 ** 58) == OVERFLOW
    assert norm_back(rows=0, dy=None, h=None, rstd=None, dx=None, dw=None) == 0
    if nodev():
        for kw in (dict(), dict(dx=A[0]), dict(dx=A[4]), dict(ds=None), dict(dw=None), dict(w=None, dw=None), dict(rows=0)):
            assert norm_back(**kw) == NODEV, kw


def adapter(X=A[0], ldx=100, Am=A[1], B=A[2], ids=A[3], scale=A[4], rows=5, m=50, n=100, k=8, count=3, prec=1, base=A[5], ldb=50,
            Y=A[6], ldy=50, hidden=A[7]):
    return L().lrc_adapter_apply(X, ldx, Am, B, ids, scale, rows, m, n, k, count, prec, base, ldb, Y, ldy, hidden)


def test_adapter_refusals():
    for kw in (dict(X=None), dict(Am=None), dict(B=None), dict(ids=None), dict(Y=None), dict(rows=-1), dict(m=0), dict(n=0),
               dict(k=0), dict(k=257), dict(count=0), dict(prec=E4M3), dict(prec=-1), dict(ldx=99), dict(ldb=49), dict(ldy=49),
               dict(Y=A[0]), dict(Y=A[1]), dict(Y=A[2]), dict(Y=A[3]), dict(Y=A[4]), dict(Y=A[5], ldy=51), dict(Y=A[5] + 2),
               dict(hidden=A[0]), dict(hidden=A[5]), dict(hidden=A[6])):
        assert adapter(**kw) == INVALID, kw
    assert adapter(rows=2 ** 23 + 1) == OVERFLOW and adapter(count=2 ** 22 + 1) == OVERFLOW and adapter(m=2 ** 31, ldb=2 ** 31, ldy=2 ** 31) == OVERFLOW
    assert adapter(ldx=2 ** 62) == OVERFLOW
    assert adapter(count=2 ** 30, n=2 ** 30, ldx=2 ** 30, k=256) == OVERFLOW
    assert adapter(rows=0, X=None, Am=None, B=None, ids=None, Y=None) == 0
    if nodev():
        for kw in (dict(), dict(Y=A[5]), dict(base=None), dict(scale=None), dict(hidden=None), dict(k=256), dict(rows=9000)):
            assert adapter(**kw) == NODEV, kw


def adapter_back(dY=A[0], lddy=50, X=A[1], ldx=100, Am=A[2], B=A[3], ids=A[4], scale=A[5], hidden=A[6], rows=5, m=50, n=100, k=8,
                 count=3, prec=1, base=A[7], ldb=100, dX=A[8], lddx=100, dA=A[9], dB=A[10]):
    return L().lrc_adapter_backward(dY, lddy, X, ldx, Am, B, ids, scale, hidden, rows, m, n, k, count, prec, base, ldb, dX, lddx,
                                    dA, dB)


def test_adapter_gradient_refusals():
    for kw in (dict(dY=None), dict(B=None), dict(ids=None), dict(Am=None), dict(X=None), dict(hidden=None), dict(rows=-1),
               dict(k=257), dict(prec=E4M3), dict(lddy=49), dict(ldx=99), dict(ldb=99), dict(lddx=99), dict(dX=A[0]), dict(dX=A[1]),
               dict(dX=A[7] + 2), dict(dX=A[7], lddx=101), dict(dX=A[6]), dict(dA=A[2]), dict(dA=A[8]), dict(dB=A[3]), dict(dB=A[9]),
               dict(dA=A[4]), dict(dB=A[7])):
        assert adapter_back(**kw) == INVALID, kw
    assert adapter_back(rows=2 ** 23 + 1) == OVERFLOW
    assert adapter_back(rows=70000, count=70000, n=2 ** 16, ldx=2 ** 16, ldb=2 ** 16, lddx=2 ** 16) == OVERFLOW
    assert b"gradients of 70000" in L().lrc_last_error()
    assert adapter_back(dX=None, dA=None, dB=None) == 0
    assert adapter_back(rows=0, dA=None, dB=None) == 0
    if nodev():
        for kw in (dict(), dict(dX=A[7]), dict(base=None), dict(dX=None, Am=None), dict(dA=None, X=None), dict(dB=None, hidden=None),
                   dict(rows=0, dY=None)):
            assert adapter_back(**kw) == NODEV, kw


def verify(logits=A[0], ld=100, lr=400, q=A[1], ldq=100, lrq=300, requests=2, drafts=3, vocab=100, prec=1, draft=A[2], u=A[3],
           t=A[4], k=A[5], p=A[6], mp=A[7], tokens=A[8], accepted=A[9]):
    return L().lrc_verify(logits, ld, lr, q, ldq, lrq, requests, drafts, vocab, prec, draft, u, t, k, p, mp, tokens, accepted)


def test_verify_refusals():
    for kw in (dict(logits=None), dict(draft=None), dict(u=None), dict(tokens=None), dict(requests=-1), dict(drafts=-1),
               dict(drafts=65537), dict(vocab=0), dict(vocab=2 ** 31, ld=2 ** 31), dict(ld=99), dict(lr=99), dict(ldq=99), dict(lrq=1),
               dict(ld=-100), dict(lr=-400), dict(prec=E4M3), dict(tokens=A[0]), dict(tokens=A[1] + 8), dict(tokens=A[2]),
               dict(tokens=A[3]), dict(accepted=A[5]), dict(accepted=A[8] + 8), dict(accepted=A[2])):
        assert verify(**kw) == INVALID, kw
    assert verify(lr=2 ** 62) == OVERFLOW and verify(requests=2 ** 62) == OVERFLOW
    assert verify(requests=0, logits=None, q=None, draft=None, u=None, tokens=None) == 0
    if nodev():
        for kw in (dict(), dict(q=None), dict(ld=0), dict(lr=0), dict(ldq=0, lrq=0), dict(t=None, k=None, p=None, mp=None),
                   dict(accepted=None), dict(drafts=0, draft=None), dict(drafts=0, q=None)):
            assert verify(**kw) == NODEV, kw


def apply8(codes=A[0], scales=A[1], sprec=2, group=32, U=A[2], s=A[3], V=A[4], k=5, fprec=2, X=A[5], ldx=100, t=A[7], Y=A[6], ldy=50,
           m=50, n=100, batch=3, yprec=1):
    return L().lrc_q4_apply_e4m3(codes, scales, sprec, group, U, s, V, k, fprec, X, ldx, t, Y, ldy, m, n, batch, yprec)


def test_8_bit_activations_refusals():
    for kw in (dict(codes=None), dict(scales=None), dict(X=None), dict(Y=None), dict(t=None), dict(U=None), dict(group=0), dict(sprec=E4M3),
               dict(fprec=E4M3), dict(yprec=E4M3), dict(k=51), dict(batch=-1), dict(ldx=99), dict(ldy=49), dict(codes=A[0] + 4),
               dict(Y=A[5]), dict(Y=A[7]), dict(Y=A[2])):
        assert apply8(**kw) == INVALID, kw
    assert apply8(batch=2 ** 60) == OVERFLOW
    assert apply8(batch=0, X=None, Y=None, t=None) == 0
    if nodev():
        assert apply8() == NODEV and apply8(k=0, U=None, s=None, V=None) == NODEV
    # the call of other types takes none of them
    assert L().lrc_q4_apply(A[0], A[1], 2, 32, None, None, None, 0, 0, A[5], 100, A[6], 50, 50, 100, 3, E4M3, 1) == INVALID


# ------------------------------------------------------------------- binding --

def test_binding_norm():
    x, w = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(8)
    for bad, match in ((lambda: lrc.rms_norm(x[0]), "matrix"), (lambda: lrc.rms_norm(x, torch.zeros(9)), "weight"),
                       (lambda: lrc.rms_norm(x, torch.zeros(16)[::2]), "weight"), (lambda: lrc.rms_norm(x, w, x.float()), "residual"),
                       (lambda: lrc.rms_norm(x, w, x[:2]), "residual"), (lambda: lrc.rms_norm(x, w, sum=x), "sum"),
                       (lambda: lrc.rms_norm(x, w, out=x.float()), ""), (lambda: lrc.rms_norm(x.t(), None), "contiguous"),
                       (lambda: lrc.rms_norm_e4m3(x, w, out=x), ""),
                       (lambda: lrc.rms_norm_backward(x, x[:2], w, torch.zeros(3)), "dy and h"),
                       (lambda: lrc.rms_norm_backward(x, x, w, None), "rstd"),
                       (lambda: lrc.rms_norm_backward(x, x, w, torch.zeros(3), dsum=x.float()), "dsum"),
                       (lambda: lrc.rms_norm_backward(x, x, w, torch.zeros(3), dx=x[:, :4]), "")):
        with pytest.raises(ValueError, match=match):
            bad()
    for bad in (lambda: lrc.rms_norm(x.double()), lambda: lrc.rms_norm(x, w.double()), lambda: lrc.rms_norm(x.to(torch.float8_e4m3fn)),
                lambda: lrc.rms_norm_backward(x, x, w, torch.zeros(3).double())):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises((ValueError, RuntimeError)):
        lrc.rms_norm(x, w)


def test_binding_adapters():
    X, Am, B = torch.zeros(4, 8), torch.zeros(2, 3, 8), torch.zeros(2, 5, 3)
    ids = torch.zeros(4, dtype=torch.int64)
    H = torch.zeros(4, 3)
    for bad in (lambda: lrc.adapter_apply(X[0], Am, B, ids), lambda: lrc.adapter_apply(X, Am[0], B, ids),
                lambda: lrc.adapter_apply(X, Am, B[:, :, :2], ids), lambda: lrc.adapter_apply(X[:, :7], Am, B, ids),
                lambda: lrc.adapter_apply(X, Am, B, None), lambda: lrc.adapter_apply(X, Am, B, ids[:3]),
                lambda: lrc.adapter_apply(X, Am, B, ids, scale=torch.zeros(3)), lambda: lrc.adapter_apply(X, Am, B, ids, base=X),
                lambda: lrc.adapter_apply(X, Am, B, ids, Y=X), lambda: lrc.adapter_apply(X, Am, B.transpose(1, 2).contiguous().transpose(1, 2), ids),
                lambda: lrc.adapter_backward(X, X, Am, B, ids, H), lambda: lrc.adapter_backward(X[:, :5], X, Am, B, ids, H[:3]),
                lambda: lrc.adapter_backward(X[:, :5], X, Am, B, ids, H.half()),
                lambda: lrc.adapter_backward(X[:, :5], X, Am, B, ids, H, base=X[:, :5])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lrc.adapter_apply(X, Am.half(), B, ids), lambda: lrc.adapter_apply(X, Am, B, ids.int()),
                lambda: lrc.adapter_apply(X, Am, B, ids, scale=torch.zeros(2).double()),
                lambda: lrc.adapter_apply(X.double(), Am.double(), B.double(), ids)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises((ValueError, RuntimeError)):
        lrc.adapter_apply(X, Am, B, ids)


def test_binding_verify():
    l, d, u = torch.zeros(2, 4, 9), torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 4)
    for bad in (lambda: lrc.verify(l[0], d, u), lambda: lrc.verify(l[:, :3], d, u), lambda: lrc.verify(l, d, u[:, :3]),
                lambda: lrc.verify(l, d, u, draft_logits=l), lambda: lrc.verify(l.transpose(1, 2).contiguous().transpose(1, 2), d, u),
                lambda: lrc.verify(l, d, u, top_p=torch.zeros(3)), lambda: lrc.verify(l, torch.zeros(2, 6, dtype=torch.int64)[:, ::2], u)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lrc.verify(l, d.int(), u), lambda: lrc.verify(l, d, u.double()), lambda: lrc.verify(l.double(), d, u),
                lambda: lrc.verify(l, d, u, draft_logits=l[:, :3].half()), lambda: lrc.verify(l, d, u, top_k=torch.zeros(2))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises((ValueError, RuntimeError)):
        lrc.verify(l, d, u)


def test_binding_8_bit_activations():
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.float16)
    X, t = torch.zeros(2, 40).to(torch.float8_e4m3fn), torch.zeros(2)
    for bad in (lambda: lrc.q4_apply(codes, scales, X, 32), lambda: lrc.q4_apply(codes, scales, X.float(), 32, x_scales=t),
                lambda: lrc.q4_apply(codes, scales, X, 32, x_scales=t[:1])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: lrc.q4_apply(codes, scales, X, 32, x_scales=t.half()),
                lambda: lrc.q4_apply(codes, scales, X, 32, x_scales=t, out_dtype=torch.float8_e4m3fn)):
        with pytest.raises((TypeError, ValueError)):
            bad()
