"""Refusals of the output-head calls, C ABI and binding (no GPU needed): every check runs before any device call."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_12969_amd import lrc  # noqa: E402

A = [0x1000000 * (i + 1) for i in range(12)]
INVALID, OVERFLOW, NODEV = -1, -2, -5


def L():
    return lrc.lib()


def nodev():
    return not torch.cuda.is_available()


def test_q4_storage():
    assert [lrc.q4_row_bytes(n) for n in (1, 32, 33, 4096)] == [16, 16, 32, 2048]
    assert lrc.q4_storage_bytes(10, 100, 64, "fp16") == 10 * 64 + 10 * 2 * 2
    assert lrc.q4_storage_bytes(10, 100, 32, "fp32") == 10 * 64 + 10 * 4 * 4
    for args in ((0, 5, 32, 1), (5, 0, 32, 1), (5, 5, 33, 1), (5, 5, 16, 1), (5, 5, 1024, 1), (5, 5, 32, 0), (5, 5, 32, 7)):
        assert L().lrc_q4_storage_bytes(*args) == INVALID
    assert L().lrc_q4_storage_bytes(2 ** 62, 2 ** 62, 32, 1) == OVERFLOW
    assert L().lrc_q4_row_bytes(0) == INVALID and L().lrc_q4_row_bytes(2 ** 63 - 1) == OVERFLOW


def quant(W=A[0], ldw=100, m=10, n=100, group=32, prec=1, codes=A[1], scales=A[2], sprec=2, values=A[3]):
    return L().lrc_q4_quantize(W, ldw, m, n, group, prec, codes, scales, sprec, values, None)


def test_q4_quantize_refusals():
    for kw in (dict(W=None), dict(codes=None), dict(scales=None), dict(ldw=99), dict(m=0), dict(n=0), dict(group=48),
               dict(prec=4), dict(sprec=0), dict(codes=A[1] + 8), dict(codes=A[0]), dict(values=A[0] + 16),
               dict(scales=A[1] + 16), dict(values=A[2] + 4)):
        assert quant(**kw) == INVALID, kw
    assert quant(m=2 ** 40, n=2 ** 40, ldw=2 ** 40) == OVERFLOW
    if nodev():
        assert quant() == NODEV and quant(values=None) == NODEV


def apply(codes=A[0], scales=A[1], sprec=2, group=32, U=A[2], s=A[3], V=A[4], k=5, fprec=2, X=A[5], ldx=100, Y=A[6], ldy=50,
          m=50, n=100, batch=3, prec=2, yprec=1):
    return L().lrc_q4_apply(codes, scales, sprec, group, U, s, V, k, fprec, X, ldx, Y, ldy, m, n, batch, prec, yprec)


def test_q4_apply_refusals():
    for kw in (dict(codes=None), dict(scales=None), dict(X=None), dict(Y=None), dict(U=None), dict(s=None), dict(V=None),
               dict(group=0), dict(sprec=0), dict(fprec=0), dict(prec=0), dict(yprec=0), dict(prec=4), dict(k=-1), dict(k=51),
               dict(batch=-1), dict(ldx=99), dict(ldy=49), dict(m=0), dict(n=0), dict(codes=A[0] + 4), dict(Y=A[0]), dict(Y=A[1]),
               dict(Y=A[2] + 2), dict(Y=A[4]), dict(Y=A[5] + 64)):
        assert apply(**kw) == INVALID, kw
    assert b"overlaps" in L().lrc_last_error()
    assert apply(batch=2 ** 60) == OVERFLOW
    assert apply(batch=0, X=None, Y=None) == 0
    if nodev():
        assert apply() == NODEV and apply(k=0, U=None, s=None, V=None) == NODEV


def sample(logits=A[0], ld=100, rows=4, vocab=100, prec=1, u=A[1], t=A[2], k=A[3], p=A[4], mp=A[5], out=A[6]):
    return L().lrc_sample(logits, ld, rows, vocab, prec, u, t, k, p, mp, out)


def test_sample_refusals():
    for kw in (dict(logits=None), dict(u=None), dict(out=None), dict(ld=99), dict(rows=-1), dict(vocab=0),
               dict(vocab=2 ** 31, ld=2 ** 31), dict(prec=0), dict(prec=4), dict(out=A[0] + 8), dict(out=A[1]), dict(out=A[3])):
        assert sample(**kw) == INVALID, kw
    assert sample(rows=2 ** 31) == OVERFLOW
    assert sample(ld=2 ** 62) == OVERFLOW
    assert sample(rows=0, logits=None, u=None, out=None) == 0
    if nodev():
        assert sample() == NODEV and sample(t=None, k=None, p=None, mp=None) == NODEV


def distill(logits=A[0], ld=100, rows=4, vocab=100, prec=1, ids=A[1], top=A[2], K=5, tprec=1, lse=A[3], w=A[4], T=1.0, loss=A[5],
            stats=A[6], grad=A[7], ldg=100):
    return L().lrc_distill(logits, ld, rows, vocab, prec, ids, top, K, tprec, lse, w, T, loss, stats, grad, ldg)


def backward(logits=A[0], ld=100, rows=4, vocab=100, prec=1, ids=A[1], top=A[2], K=5, tprec=1, lse=A[3], w=A[4], T=1.0,
             stats=A[6], dloss=A[5], grad=A[7], ldg=100):
    return L().lrc_distill_backward(logits, ld, rows, vocab, prec, ids, top, K, tprec, lse, w, T, stats, dloss, grad, ldg)


def test_distill_refusals():
    both = (dict(logits=None), dict(ids=None), dict(top=None), dict(ld=99), dict(rows=-1), dict(vocab=0), dict(prec=0), dict(tprec=0),
            dict(K=0), dict(K=1025), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-300),
            dict(ldg=99), dict(grad=A[0] + 4), dict(grad=A[0], ldg=101), dict(grad=A[1]), dict(grad=A[2]), dict(grad=A[4]))
    for kw in both + (dict(loss=None), dict(loss=A[0] + 4), dict(stats=A[5]), dict(loss=A[7] + 8), dict(stats=A[3])):
        assert distill(**kw) == INVALID, kw
    for kw in both + (dict(stats=None), dict(grad=None), dict(grad=A[6]), dict(grad=A[5])):
        assert backward(**kw) == INVALID, kw
    assert distill(rows=2 ** 31) == OVERFLOW and backward(ld=2 ** 62) == OVERFLOW
    assert distill(rows=0, logits=None, ids=None, top=None, loss=None, stats=None, grad=None) == 0
    if nodev():
        for f in (distill, backward):
            assert f() == NODEV and f(grad=A[0]) == NODEV and f(lse=None, w=None) == NODEV
        assert distill(grad=None, ldg=0) == NODEV and backward(dloss=None) == NODEV


def test_factor_calls_keep_refusing_bfloat16():
    good = [0x10000, 0x20000, 0x30000, 0x40000, 0x90000000]
    assert L().lrc_matrix_apply(*good, 10, 10, 3, 4, lrc.BF16) == INVALID
    with pytest.raises(TypeError):
        lrc.matrix_apply(*[torch.zeros(3, 3, dtype=torch.bfloat16)] * 4)


# ------------------------------------------------------------------- binding --

def test_binding_q4_checks():
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.float16)
    X = torch.zeros(2, 40, dtype=torch.float16)
    with pytest.raises(ValueError, match="shape mismatch"):
        lrc.q4_apply(codes, scales, X, 64)
    with pytest.raises(ValueError, match="shape mismatch"):
        lrc.q4_apply(codes, scales, torch.zeros(2, 70, dtype=torch.float16), 32)
    with pytest.raises(TypeError, match="uint8"):
        lrc.q4_apply(codes.int(), scales, X, 32)
    with pytest.raises(TypeError, match="float64"):
        lrc.q4_apply(codes, scales, X.double(), 32)
    with pytest.raises(TypeError, match="float64"):
        lrc.q4_apply(codes, scales.double(), X, 32)
    with pytest.raises(ValueError, match="contiguous"):
        lrc.q4_apply(codes, scales, torch.zeros(40, 2, dtype=torch.float16).t(), 32)
    with pytest.raises(ValueError, match="Y has shape"):
        lrc.q4_apply(codes, scales, X, 32, Y=torch.zeros(2, 9))
    with pytest.raises(ValueError, match="Y has dtype"):
        lrc.q4_apply(codes, scales, X, 32, out_dtype=torch.float32, Y=torch.zeros(2, 8, dtype=torch.float16))
    F = (torch.zeros(8, 3), torch.zeros(3), torch.zeros(40, 3))
    with pytest.raises(ValueError, match="shape mismatch"):
        lrc.q4_apply(codes, scales, X, 32, (F[0], F[1], torch.zeros(41, 3)))
    with pytest.raises(TypeError, match="one dtype"):
        lrc.q4_apply(codes, scales, X, 32, (F[0].half(), F[1], F[2]))
    with pytest.raises(ValueError, match="on the GPU"):
        lrc.q4_apply(codes, scales, X, 32, F)
    with pytest.raises(ValueError, match="group"):
        lrc.q4_quantize(torch.zeros(3, 3), 48)
    with pytest.raises(ValueError, match="on the GPU"):
        lrc.q4_quantize(torch.zeros(3, 3), 32)
    with pytest.raises(ValueError, match="matrix"):
        lrc.q4_quantize(torch.zeros(3), 32)


def test_binding_sample_checks():
    l, u = torch.zeros(3, 10), torch.zeros(3)
    with pytest.raises(ValueError, match="u must"):
        lrc.sample(l, torch.zeros(4))
    with pytest.raises(TypeError, match="u has"):
        lrc.sample(l, u.double())
    with pytest.raises(TypeError, match="top_k"):
        lrc.sample(l, u, top_k=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="top_p"):
        lrc.sample(l, u, top_p=torch.zeros(3, 1))
    with pytest.raises(TypeError):
        lrc.sample(l.double(), u)
    with pytest.raises(ValueError, match="contiguous"):
        lrc.sample(torch.zeros(10, 3).t(), u)
    with pytest.raises(ValueError, match="on the GPU"):
        lrc.sample(l, u)


def test_binding_distill_checks():
    z, ids, top = torch.zeros(3, 10), torch.zeros(3, 2, dtype=torch.int64), torch.zeros(3, 2)
    for f in (lrc.distill, lrc.distill_forward):
        with pytest.raises(TypeError, match="ids"):
            f(z, ids.int(), top)
        with pytest.raises(ValueError, match="shape mismatch"):
            f(z, ids, torch.zeros(3, 3))
        with pytest.raises(ValueError, match="shape mismatch"):
            f(z, ids[:2], top[:2])
        with pytest.raises(ValueError, match="weight"):
            f(z, ids, top, weight=torch.zeros(2))
        with pytest.raises(TypeError, match="teacher_lse"):
            f(z, ids, top, teacher_lse=torch.zeros(3, dtype=torch.float64))
        with pytest.raises(ValueError, match="on the GPU"):
            f(z, ids, top)
