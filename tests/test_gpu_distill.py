"""Distillation loss and gradient against the binary64 oracle (oracle/head.py).

Tolerances.  exp of a difference of logits carries a relative error of a few 2^-24 plus the rounding of its argument,
|z - max| / T <= 40 here: 40 * 2^-23 = 5e-6 at most, for terms that size has made negligible; sums of positive terms keep
that.  So q is held to 1e-5, the loss to 1e-5 of its terms' size w T^2 (|loss| + 1), a gradient entry to 1e-5 w T (q + p)
plus one rounding to its type."""
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


def case(seed, rows, V, K, prec, T, tail, tprec="fp32"):
    rng = np.random.default_rng(seed)
    teacher = rng.normal(size=(rows, V)) * 2.5
    z = torch.from_numpy(teacher + 0.5 * rng.normal(size=(rows, V))).to(DT[prec]).cuda()
    ids = np.argsort(-teacher, 1)[:, :K].copy()
    if ids.shape[1] < K:
        ids = np.pad(ids, ((0, 0), (0, K - ids.shape[1])), constant_values=-1)
    top = torch.from_numpy(np.take_along_axis(teacher, np.maximum(ids, 0), 1)).to(DT[tprec]).cuda()
    lse = np.log(np.exp(teacher / T).sum(1)).astype(np.float32)
    for r in range(1, rows, 3):                           # rows that know fewer tokens, slots in any place
        ids[r, rng.random(K) < 0.5] = rng.choice([-1, V, V + 100, -2 ** 40])
    w = rng.random(rows).astype(np.float32) + 0.5
    w[::4] = 0 if rows > 3 else w[::4]
    return (z, torch.from_numpy(ids).cuda(), top, torch.from_numpy(lse).cuda() if tail else None,
            torch.from_numpy(w).cuda())


def reference(z, ids, top, T, lse, w):
    n = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    return H.distill(n(z), ids.cpu().numpy(), n(top), float(np.float32(T)), n(lse), n(w))


def near(loss, grad, want_loss, want_grad, z, ids, T, w, prec, up=1.0):
    w = np.ones(len(want_loss)) if w is None else w.double().cpu().numpy()
    if loss is not None:
        err = abs(loss.double().cpu().numpy() - want_loss)
        assert (err <= 1e-5 * (abs(want_loss) + w * T * T)).all(), float(err.max())
    if grad is not None:
        x = z.double().cpu().numpy() / T
        q = np.exp(x - x.max(1, keepdims=True))
        q /= q.sum(1, keepdims=True)
        size = (w * T)[:, None] * q
        want = want_grad * up
        tol = 1e-5 * (2 * size * up + abs(want)) + UNIT[prec] * abs(want) + TINY[prec]
        got = grad.double().cpu().numpy()
        assert (abs(got - want) <= tol).all(), float((abs(got - want) / tol).max())


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,V,K,T", [(1, 1, 1, 1.0), (2, 3, 2, 2.0), (5, 64, 7, 1.0), (9, 1001, 64, 4.0), (3, 4099, 1000, 1.0),
                                        (13, 32003, 33, 2.0), (2, 70001, 256, 1.0), (2, 131072, 16, 1.0), (2, 300007, 50, 1.5)])
def test_distill_matches_oracle(lrc, prec, tail, rows, V, K, T):
    z, ids, top, lse, w = case(V + K, rows, V, min(K, V) if V < 4 else K, prec, T, tail)
    L, G = reference(z, ids, top, T, lse, w)
    kw = dict(temperature=T, teacher_lse=lse, weight=w)
    loss, grad = lrc.distill(z, ids, top, **kw)
    near(loss, grad, L, G, z, ids, T, w, prec)
    again = lrc.distill(z, ids, top, **kw)
    assert torch.equal(loss, again[0]) and torch.equal(grad, again[1])
    floss, stats = lrc.distill_forward(z, ids, top, **kw)
    near(floss, None, L, G, z, ids, T, w, prec)
    near(None, lrc.distill_backward(z, ids, top, stats, **kw), L, G, z, ids, T, w, prec)
    up = torch.rand(rows, device="cuda") + 0.5
    g = lrc.distill_backward(z, ids, top, stats, dloss=up, **kw)
    near(None, g, L, G, z, ids, T, w, prec, up.double().cpu().numpy()[:, None])


def test_distill_gradient_against_differences(lrc):
    """Differences of the kernel's own loss: with step h an error of 1e-6 (loss rounding) / h + h^2 / 6."""
    z, ids, top, lse, w = case(3, 6, 11, 4, "fp32", 1.5, True)
    kw = dict(temperature=1.5, teacher_lse=lse, weight=w)
    _, grad = lrc.distill(z, ids, top, **kw)
    h = 2.0 ** -6
    for j in range(11):
        d = torch.zeros_like(z)
        d[:, j] = h
        num = (lrc.distill_forward(z + d, ids, top, **kw)[0] - lrc.distill_forward(z - d, ids, top, **kw)[0]) / (2 * h)
        assert (num - grad[:, j]).abs().max() < 1e-3


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("tprec", ["fp32", "fp16", "bf16"])
def test_distill_teacher_types_pitches_in_place(lrc, prec, tprec):
    T = 1.0
    z, ids, top, lse, w = case(11, 7, 1003, 20, prec, T, True, tprec)
    lse = lse + 0.05                                      # the stored logits' rounding must not pass the whole mass
    L, G = reference(z, ids, top, T, lse, w)
    big = torch.full((7, 1100), float("nan"), dtype=DT[prec], device="cuda")
    for off in (0, 8, 3):
        part = big[:, off:off + 1003]
        part.copy_(z)
        loss, grad = lrc.distill(part, ids, top, teacher_lse=lse, weight=w)
        near(loss, grad, L, G, z, ids, T, w, prec)
        _, stats = lrc.distill_forward(part, ids, top, teacher_lse=lse, weight=w)
        loss2, same = lrc.distill(part, ids, top, teacher_lse=lse, weight=w, grad=part)
        assert same is part and torch.equal(part, grad) and torch.equal(loss, loss2)
        part.copy_(z)
        lrc.distill_backward(part, ids, top, stats, teacher_lse=lse, weight=w, grad=part)
        near(None, part, L, G, z, ids, T, w, prec)
        assert big[:, :off].isnan().all() and big[:, off + 1003:].isnan().all()
        big.fill_(float("nan"))


def test_distill_tokens_named_twice(lrc):
    z, ids, top, _, _ = case(5, 4, 50, 6, "fp32", 1.0, False)
    ids[0, 1] = ids[0, 0]
    ids[1, :] = 7
    ids[2, 5] = ids[2, 2]
    for lse in (None, torch.full((4,), 12.0, device="cuda")):
        L, G = reference(z, ids, top, 1.0, lse, None)
        loss, grad = lrc.distill(z, ids, top, teacher_lse=lse)
        near(loss, grad, L, G, z, ids, 1.0, None, "fp32")


def test_distill_rows_that_name_or_count_nothing(lrc):
    z, ids, top, lse, _ = case(6, 5, 333, 8, "bf16", 1.0, True)
    ids[0] = -1
    top[1] = float("-inf")
    w = torch.ones(5, device="cuda")
    w[2] = 0
    z[2] = float("nan")
    for t in (None, lse):
        loss, grad = lrc.distill(z, ids, top, teacher_lse=t, weight=w)
        assert loss[2] == 0 and not grad[2].any()
        if t is None:
            assert loss[0] == 0 and loss[1] == 0 and not grad[:2].any()
        else:
            assert abs(loss[0].item()) < 1e-6 and grad[0].abs().max() < 1e-6     # all mass in the other class
        assert loss.isfinite().all() and grad.isfinite().all()
        _, stats = lrc.distill_forward(z, ids, top, teacher_lse=t, weight=w)
        back = lrc.distill_backward(z, ids, top, stats, teacher_lse=t, weight=w)
        assert not back[2].any() and back.isfinite().all()


def test_distill_masked_and_extreme_logits(lrc):
    V = 2000
    z = torch.randn(6, V, device="cuda")
    z[:, 1000:] = float("-inf")                          # forbidden by a mask
    z[1, :1000] = torch.finfo(torch.float32).min         # the type's lowest value beside one real logit
    z[1, 3] = 1.0
    z[2] = float("-inf")                                 # nothing left
    z[3, 5] = float("nan")
    z[4] = 1e4 * torch.randn(V, device="cuda")           # far apart
    z[5, :4] = 200.0                                     # all the student's mass on named tokens
    ids = torch.tensor([[3, 1, 2, 0]] * 6, device="cuda")
    ids[4] = z[4].topk(4).indices
    top = torch.tensor([[2.0, 1.0, 0.5, 0.0]] * 6, device="cuda")
    lse = torch.logsumexp(top, 1) + 0.1
    for t in (None, lse):
        loss, grad = lrc.distill(z, ids, top, teacher_lse=t)
        assert loss[2].isnan() and loss[3].isnan() and grad[2].isnan().all() and grad[3].isnan().all()
        rows = [0, 4, 5]
        L, G = reference(z[rows], ids[rows], top[rows], 1.0, None if t is None else t[rows], None)
        got = loss[rows].double().cpu().numpy()
        same = (got == L) | (abs(got - L) <= 1e-5 * (1 + abs(L)))
        assert same.all(), (got, L)
        fin = np.isfinite(L)
        near(None, grad[rows][torch.from_numpy(fin).cuda()], None, G[fin], z[rows][torch.from_numpy(fin).cuda()], None, 1.0,
             torch.ones(int(fin.sum())), "fp32") if fin.any() else None
        assert not grad[0, 1000:].any() and loss[1] > 1e30
    # a named token that the student gives -infinity
    z = torch.zeros(1, 10, device="cuda")
    z[0, 4] = float("-inf")
    loss, grad = lrc.distill(z, torch.tensor([[4]], device="cuda"), torch.zeros(1, 1, device="cuda"))
    assert loss.item() == float("inf") and grad[0, 4] == -1.0


def test_distill_named_token_without_teacher_mass(lrc):
    z = torch.randn(2, 40, device="cuda")
    ids = torch.tensor([[1, 2], [5, 6]], device="cuda")
    top = torch.tensor([[0.3, float("-inf")], [0.1, 0.2]], device="cuda")
    for lse in (None, torch.tensor([1.0, 1.5], device="cuda")):
        L, G = reference(z, ids, top, 1.0, lse, None)
        loss, grad = lrc.distill(z, ids, top, teacher_lse=lse)
        near(loss, grad, L, G, z, ids, 1.0, None, "fp32")


def test_distill_zero_rows_and_stream(lrc):
    e = torch.empty(0, 5, device="cuda")
    loss, grad = lrc.distill(e, torch.empty(0, 2, dtype=torch.int64, device="cuda"), torch.empty(0, 2, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, 5)
    z, ids, top, lse, w = case(8, 5, 777, 9, "bf16", 1.0, True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        a = lrc.distill(z, ids, top, teacher_lse=lse, weight=w)
    st.synchronize()
    b = lrc.distill(z, ids, top, teacher_lse=lse, weight=w)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
