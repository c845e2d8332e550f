"""4-bit products of more rows than one panel of 2^20 takes, against binary64 products of the same stored values.

Tolerance: with u = 2^-24, (n + n / group + 8) u (|X| |W|^T) for the sums, (n + k + 8) u (|X| |V| |s| |U|^T) for the
compensation, half an ulp of the stored type (2^-11 |Y|, 2^-24 below the normal range)."""
import numpy as np
import pytest

from oracle import head as H

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("batch", [2 ** 20, 2 ** 20 + 1, 2 ** 21, 2 ** 21 + 37])
@pytest.mark.parametrize("n,k", [(32, 0), (200, 5)])
def test_product_of_many_rows(lrc, batch, n, k):
    rng = np.random.default_rng(n + k)
    m, group, u = 16, 32, 2.0 ** -24
    codes = rng.integers(0, 16, (m, n))
    scales = torch.from_numpy(0.05 * (0.25 + rng.random((m, -(-n // group))))).half()
    W = torch.from_numpy(H.weights(codes, scales.double().numpy(), group)).cuda()
    packed, scales = torch.from_numpy(H.pack(codes)).cuda(), scales.cuda()
    g = torch.Generator(device="cuda").manual_seed(batch)
    X = torch.randn(batch, n, generator=g, device="cuda", dtype=torch.float16)
    F = None
    if k:
        F = tuple(torch.randn(*s, generator=g, device="cuda", dtype=torch.float16) for s in ((m, k), (k,), (n, k)))
    Y = lrc.q4_apply(packed, scales, X, group, F)
    for b0 in range(0, batch, 2 ** 18):
        x = X[b0:b0 + 2 ** 18].double()
        ref, bound = x @ W.t().contiguous(), (n + n / group + 8) * u * (x.abs() @ W.abs().t().contiguous())
        if k:
            U, s, V = (f.double() for f in F)
            ref += ((x @ V) * s) @ U.t().contiguous()
            bound += (n + k + 8) * u * (((x.abs() @ V.abs()) * s.abs()) @ U.abs().t().contiguous())
        bound += 2.0 ** -11 * ref.abs() + 2.0 ** -24
        assert ((Y[b0:b0 + 2 ** 18].double() - ref).abs() <= bound).all(), b0
