"""Tokens that a teacher names twice, in every kernel of the distillation loss: the one-pass step with its row in
registers and its row read again, the loss alone and the gradient alone, whose rows are taken in slabs of 2^18 logits."""
import numpy as np
import pytest

from test_gpu_distill_contract import check, up  # noqa: F401
from oracle import head as H

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("V", [50, 5003, 70001, 300007])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows", [4, 1030])
def test_duplicates_in_every_kernel(lrc, prec, V, tail, rows):
    if rows * V > 10 ** 7:
        rows = 5
    rng = np.random.default_rng(V)
    K, T = 6, 1.0
    teacher = 2.0 * rng.normal(size=(rows, V))
    z = torch.from_numpy(teacher + 0.5 * rng.normal(size=(rows, V))).to(DT[prec]).cuda()
    ids = np.argsort(-teacher, 1)[:, :K].copy()
    ids[0::4, :3] = 0                                    # first and last place of the row: the ends of its slabs
    ids[0::4, 3:5] = V - 1
    ids[1::4, 5] = ids[1::4, 0]
    ids[2::4, :] = ids[2::4, :1]
    top = torch.from_numpy(np.take_along_axis(teacher, ids, 1)).float().cuda()
    p = np.exp(up(top))
    lse = torch.from_numpy(np.log(p.sum(1) / 0.7).astype(np.float32)).cuda()     # 0.7 of the mass is named
    w = torch.from_numpy((rng.random(rows) + 0.5).astype(np.float32)).cuda()
    ids = torch.from_numpy(ids).cuda()
    full = torch.from_numpy(np.log(p.sum(1))).cuda()     # what renormalizing divides by
    kw = dict(temperature=T, teacher_lse=lse if tail else None, weight=w)
    loss, grad = lrc.distill(z, ids, top, **kw)
    floss, stats = lrc.distill_forward(z, ids, top, **kw)
    back = lrc.distill_backward(z, ids, top, stats, **kw)
    if tail:
        check(loss, grad, z, ids, top, T, lse, w, prec)
        check(floss, back, z, ids, top, T, lse, w, prec)
        return
    L, G = H.distill(up(z), ids.cpu().numpy(), up(top), T, None, up(w))
    q = np.exp(up(z) - up(z).max(1, keepdims=True))
    size = q / q.sum(1, keepdims=True)
    np.add.at(size, (np.arange(rows)[:, None], ids.cpu().numpy()), np.exp(up(top) - up(full)[:, None]))
    unit = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[prec]
    tol = 1e-5 * up(w)[:, None] * size + unit * abs(G) + (2.0 ** -25 if prec == "fp16" else 1e-38)
    for l, g in ((loss, grad), (floss, back)):
        assert (abs(up(l) - L) <= 1e-5 * (abs(L) + up(w))).all()
        assert (abs(up(g) - G) <= tol).all()
