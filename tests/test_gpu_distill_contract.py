"""What the interface says of the distillation loss beyond the common case, against the binary64 oracle.

Tolerances.  A probability of the student is held to 1e-5 of itself (a few 2^-24 and the rounding of its argument, at most
40 here), one of the teacher to a few 2^-24 of itself, so a gradient entry to 1e-5 w T (mass q + p) plus one rounding to its
type, mass being the sum of the teacher's classes; the loss to 1e-5 of its terms' size w T^2 (|loss| + mass)."""
import numpy as np
import pytest

from oracle import head as H

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 1e-38, "fp16": 2.0 ** -25, "bf16": 1e-38}


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def up(t):
    return t.double().cpu().numpy()


def heavy(seed, rows, V, K, prec, tprec, T):
    """Teachers whose named probabilities sum above 1: by a lse of other logits than the stored ones, by the stored
    logits' rounding, by a token named twice.  Every fourth row stays below 1."""
    rng = np.random.default_rng(seed)
    teacher = 2.5 * rng.normal(size=(rows, V))
    z = torch.from_numpy(teacher + 0.5 * rng.normal(size=(rows, V))).to(DT[prec]).cuda()
    ids = np.argsort(-teacher, 1)[:, :K].copy()
    ids[2::4, 1] = ids[2::4, 0]
    top = torch.from_numpy(np.take_along_axis(teacher, ids, 1)).to(DT[tprec]).cuda()
    lse = np.log(np.exp(teacher / T).sum(1))
    named = np.exp(np.take_along_axis(teacher, ids, 1) / T - lse[:, None]).sum(1)
    lse[0::4] += np.log(named[0::4]) - 0.4               # sums of about 1.5
    lse[1::4] += np.log(named[1::4])                     # about 1, by rounding above or below
    lse[2::4] += np.log(named[2::4]) - 0.1
    lse[3::4] += 0.5
    w = torch.from_numpy((rng.random(rows) + 0.5).astype(np.float32)).cuda()
    return z, torch.from_numpy(ids).cuda(), top, torch.from_numpy(lse.astype(np.float32)).cuda(), w


def check(loss, grad, z, ids, top, T, lse, w, prec, scale=None):
    host_w = up(w) if scale is None else up(w) * up(scale)
    L, _ = H.distill(up(z), ids.cpu().numpy(), up(top), T, up(lse), up(w))
    _, G = H.distill(up(z), ids.cpu().numpy(), up(top), T, up(lse), host_w)
    p = np.exp(up(top) / T - up(lse)[:, None])
    mass = np.maximum(p.sum(1), 1.0)
    if loss is not None:
        assert (abs(up(loss) - L) <= 1e-5 * up(w) * T * T * (abs(L) / (up(w) * T * T) + mass)).all()
    if grad is not None:
        q = np.exp(up(z) / T - (up(z) / T).max(1, keepdims=True))
        size = mass[:, None] * q / q.sum(1, keepdims=True)
        np.add.at(size, (np.arange(len(p))[:, None], ids.cpu().numpy()), p)
        tol = 1e-5 * (host_w * T)[:, None] * size + UNIT[prec] * abs(G) + TINY[prec]
        assert (abs(up(grad) - G) <= tol).all(), float((abs(up(grad) - G) / tol).max())


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("tprec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,V,K,T", [(8, 200, 64, 1.0), (5, 1001, 20, 2.0), (4, 70001, 40, 1.0), (4, 300007, 9, 1.5)])
def test_named_probabilities_above_one(lrc, prec, tprec, rows, V, K, T):
    z, ids, top, lse, w = heavy(V + K, rows, V, K, prec, tprec, T)
    kw = dict(temperature=T, teacher_lse=lse, weight=w)
    loss, grad = lrc.distill(z, ids, top, **kw)
    check(loss, grad, z, ids, top, T, lse, w, prec)
    loss, stats = lrc.distill_forward(z, ids, top, **kw)
    check(loss, None, z, ids, top, T, lse, w, prec)
    check(None, lrc.distill_backward(z, ids, top, stats, **kw), z, ids, top, T, lse, w, prec)
    scale = torch.rand(rows, device="cuda") + 0.5
    check(None, lrc.distill_backward(z, ids, top, stats, dloss=scale, **kw), z, ids, top, T, lse, w, prec, scale)


def test_named_probabilities_above_one_against_differences(lrc):
    """Differences of the kernel's own loss: 1e-6 of loss rounding over the step, and the third derivative's h^2 / 6."""
    z, ids, top, lse, w = heavy(3, 8, 11, 4, "fp32", "bf16", 1.5)
    kw = dict(temperature=1.5, teacher_lse=lse, weight=w)
    _, grad = lrc.distill(z, ids, top, **kw)
    h = 2.0 ** -6
    for j in range(11):
        d = torch.zeros_like(z)
        d[:, j] = h
        num = (lrc.distill_forward(z + d, ids, top, **kw)[0] - lrc.distill_forward(z - d, ids, top, **kw)[0]) / (2 * h)
        assert (num - grad[:, j]).abs().max() < 1e-3
    assert grad.double().sum(1).abs().max() < 1e-4       # the entries' tolerances summed: 1e-5 w T 2 mass


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("V", [1, 203, 20011, 70001, 300007])
@pytest.mark.parametrize("tail", [False, True])
def test_one_call_gives_loss_statistics_and_gradient(lrc, prec, V, tail):
    """The C entry with all three outputs: the statistics are those that the gradient alone takes."""
    rows, K, T = 5, min(V, 7), 1.5
    z, ids, top, lse, w = heavy(V, rows, V, K, prec, "fp32", T) if V > 1 else (
        torch.ones(rows, 1, dtype=DT[prec], device="cuda"), torch.zeros(rows, 1, dtype=torch.int64, device="cuda"),
        torch.ones(rows, 1, device="cuda"), torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda"))
    w[3] = 0                                             # a row that does not count
    ids[4] = -1                                          # a teacher that names nothing
    lse = lse if tail else None
    kw = dict(temperature=T, teacher_lse=lse, weight=w)
    grad = torch.empty_like(z)
    loss, stats = torch.empty(rows, device="cuda"), torch.full((rows, 4), float("nan"), device="cuda")
    code = {"fp32": lrc.FP32, "fp16": lrc.FP16, "bf16": lrc.BF16}
    lrc.lib().lrc_set_stream(torch.cuda.current_stream().cuda_stream)
    assert lrc.lib().lrc_distill(z.data_ptr(), V, rows, V, code[prec], ids.data_ptr(), top.data_ptr(), K, lrc.FP32,
                                 lse.data_ptr() if tail else None, w.data_ptr(), T, loss.data_ptr(), stats.data_ptr(),
                                 grad.data_ptr(), V) == 0
    want_loss, want_stats = lrc.distill_forward(z, ids, top, **kw)
    # the two calls sum a row in their own fixed orders; w T^2 (|loss| + mass) is below 10, w T 2 mass below 7
    assert torch.allclose(loss, want_loss, rtol=0, atol=1e-4)
    assert torch.allclose(stats, want_stats, rtol=1e-5, atol=0)
    back = lrc.distill_backward(z, ids, top, stats, **kw)
    assert torch.allclose(back.float(), grad.float(), rtol=2.1 * UNIT[prec], atol=1.4e-4)


@pytest.mark.parametrize("V", [50, 40000])
def test_teacher_that_names_only_nan(lrc, V):
    """A NaN among the named teacher logits makes the row's loss NaN, beside other values or alone."""
    z = torch.randn(4, V, device="cuda")
    ids = torch.tensor([[1, 2, 3]] * 4, device="cuda")
    top = torch.tensor([[1.0, 0.5, 0.0]] * 4, device="cuda")
    top[1] = float("nan")
    top[2, 1] = float("nan")
    top[3] = float("nan")
    ids[3, :] = -1                                       # NaN in unused slots does not count
    for lse in (None, torch.full((4,), 2.0, device="cuda")):
        loss, grad = lrc.distill(z, ids, top, teacher_lse=lse)
        floss, stats = lrc.distill_forward(z, ids, top, teacher_lse=lse)
        back = lrc.distill_backward(z, ids, top, stats, teacher_lse=lse)
        for x in (loss, floss):
            assert x[[0, 3]].isfinite().all() and x[1].isnan() and x[2].isnan()
        for x in (grad, back):
            assert x[[0, 3]].isfinite().all() and x[1, 1:4].isnan().all() and x[2, 1:4].isnan().all()


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,V,K,T", [(9, 1000, 1, 4.0), (7, 30001, 4, 4.0), (5, 131072, 4, 4.0), (3, 131072, 200, 4.0),
                                        (3, 300007, 3, 2.0), (6, 5000, 64, 1.0)])
def test_loss_of_little_named_mass(lrc, prec, rows, V, K, T):
    """Where the rest of both distributions is nearly all of them, the loss is what its terms leave: sum p log(p / q) and
    r log(r / Q) cancel to the square of their size.  Named tokens lie within 8 / log2(e) of the maximum here, so their q is
    right to 5e-7 and p, the logarithms to a few 2^-24: an error of 2e-6 (sum p (1 + |log p / q|) + sum q), whatever the
    sum over the row, whose error the two terms share."""
    rng = np.random.default_rng(V + K)
    teacher = rng.normal(size=(rows, V))
    z = torch.from_numpy(teacher + 0.5 * rng.normal(size=(rows, V))).to(DT[prec]).cuda()
    ids = np.argsort(-teacher, 1)[:, :K].copy()
    top = torch.from_numpy(np.take_along_axis(teacher, ids, 1)).float().cuda()
    lse = torch.from_numpy(np.log(np.exp(teacher / T).sum(1)).astype(np.float32)).cuda()
    ids = torch.from_numpy(ids).cuda()
    L, _ = H.distill(up(z), ids.cpu().numpy(), up(top), T, up(lse))
    x = up(z) / T
    q = np.take_along_axis(np.exp(x - x.max(1, keepdims=True)), ids.cpu().numpy(), 1)
    q /= np.exp(x - x.max(1, keepdims=True)).sum(1, keepdims=True)
    p = np.exp(up(top) / T - up(lse)[:, None])
    tol = 2e-6 * T * T * ((p * (1 + abs(np.log(p / q)))).sum(1) + q.sum(1)) + 2.0 ** -24 * abs(L)
    loss, _ = lrc.distill(z, ids, top, temperature=T, teacher_lse=lse)
    floss, _ = lrc.distill_forward(z, ids, top, temperature=T, teacher_lse=lse)
    for l in (loss, floss):
        assert (abs(up(l) - L) <= tol).all(), float((abs(up(l) - L) / tol).max())
