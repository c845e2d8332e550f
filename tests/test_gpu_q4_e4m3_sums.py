"""Sums of the 4-bit product of 8-bit activations where its results are FP16 or FP32: binary32, whatever the range of the
activations, also where large products cancel."""
import numpy as np
import pytest

from oracle import head as H
from test_gpu_q4_e4m3_tiles import DT, E4M3, SIZES, check, problem, some, weights

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("prec", ["fp16", "fp32"])
@pytest.mark.parametrize("b", [1, 8, 9, 16, 40, 64, 130, 2100])
@pytest.mark.parametrize("m,n,group", [(300, 1024, 128), (8192, 1000, 512), (260, 1040, 32), (70, 777, 64)])
def test_small_products_beside_large_ones_that_cancel(lrc, prec, b, m, n, group):
    """Each eight columns hold 448 * 6 (or its negative in the next eight) and seven products of 0.1171875: whole multiples
    of 2^-7 whose sums stay below 2^15, so binary32 holds every partial sum, in any order; 7 * 0.1171875 * n / 8 rounds to
    the result's type."""
    nib = np.ones((m, n), int)
    nib[:, 0::16], nib[:, 8::16] = 7, 15
    if n // 8 % 2:
        nib[:, n // 8 * 8 - 8] = 1                                   # one without a partner: left small
    if n % 8:
        nib[:, n // 8 * 8] = 1
    x = torch.full((b, n), 0.234375)
    x[:, 0::8] = torch.where(torch.from_numpy(nib[0, 0::8] == 1), 0.234375, 448.0)
    nib[1::2] ^= 8                                                   # odd rows: all signs changed
    X, t = x.to(E4M3).cuda(), torch.tensor([2.0 ** (i % 5 - 3) for i in range(b)], device="cuda")
    W = H.weights(nib, np.ones((m, -(-n // group))), group)
    want = x.double().numpy()[:1] @ W.T
    assert (np.abs(want) == 0.234375 / 2 * (x[0] < 1).sum().item()).all()
    want = torch.from_numpy(want).cuda() * t[:, None].double()
    got = lrc.q4_apply(torch.from_numpy(H.pack(nib)).cuda(), torch.ones(m, -(-n // group), device="cuda"), X, group,
                       out_dtype=DT[prec], x_scales=t)
    assert torch.equal(got, want.to(DT[prec]))


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("sdt,fdt", [("fp16", "fp16"), ("fp32", "bf16")])
def test_every_binade(lrc, size, sdt, fdt):
    m, n, k, group, b = size
    nib, codes, scales, X, t, F = problem(4, b, m, n, k, group, sdt, fdt, True)
    rng = np.random.default_rng([m, n, b])
    rows, cols = some(rng, b, (0, 15, 64, 255)), some(rng, m, (0, 63, 128, 256))
    ri, ci = torch.from_numpy(rows).cuda(), torch.from_numpy(cols).cuda()
    for prec in ("fp16", "fp32"):
        got = lrc.q4_apply(codes, scales, X, group, F, out_dtype=DT[prec], x_scales=t)
        check(got[ri][:, ci], weights(nib, scales, n, group, cols), X.view(torch.uint8)[ri].view(E4M3), t[ri], (F[0][ci], F[1], F[2]),
              prec, False)
