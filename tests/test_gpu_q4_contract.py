"""What the interface says of the 4-bit product and quantization beyond the common case."""
import numpy as np
import pytest

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


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("fprec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("b", [1, 5, 20])
@pytest.mark.parametrize("k", [1, 33, 90])
def test_infinite_activations_through_the_compensation(lrc, prec, fprec, b, k):
    """Weights, U and s above 0 and one sign a row of V: an infinity gives the infinity of the sums, not NaN; and the
    other rows are those of the call without it."""
    rng = np.random.default_rng(b + k)
    m, n = 96, 200
    codes = torch.from_numpy(H.pack(rng.integers(1, 8, (m, n)))).cuda()
    scales = torch.ones(m, -(-n // 32), dtype=torch.float16, device="cuda")
    sign = torch.ones(n, 1)
    sign[1::2] = -1
    mixed = torch.from_numpy(1.0 + rng.random((n, k))).float()
    mixed[::3] = 1.0                                     # one significant bit: what a split leaves is 0
    U, s, V = (x.to(DT[fprec]).cuda() for x in (1.0 + torch.rand(m, k), torch.ones(k), mixed * sign))
    X = torch.from_numpy(rng.random((b, n))).to(DT[prec]).cuda()
    clean = lrc.q4_apply(codes, scales, X, 32, (U, s, V), out_dtype=torch.float32)
    assert clean.isfinite().all()
    for j, want in ((0, np.inf), (3, None), (7, None), (6, np.inf), (199, None)):
        Z = X.clone()
        Z[b - 1, j] = float("inf")
        Y = lrc.q4_apply(codes, scales, Z, 32, (U, s, V), out_dtype=torch.float32)
        assert torch.equal(Y[:b - 1], clean[:b - 1])
        if want is None:                                 # + infinity from W, - infinity from the compensation
            assert Y[b - 1].isnan().all()
        else:
            assert (Y[b - 1] == want).all(), (prec, fprec, j)
    Z[b - 1, 199] = float("nan")
    Y = lrc.q4_apply(codes, scales, Z, 32, (U, s, V), out_dtype=torch.float32)
    assert torch.equal(Y[:b - 1], clean[:b - 1]) and Y[b - 1].isnan().all()


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32", "fp64"])
def test_groups_of_scale_zero_keep_their_signs(lrc, prec):
    """Weights too small for the scale's type: magnitude 0, the weight's sign; a group of scale NaN: codes 0."""
    tiny = 2.0 ** -24 if prec == "fp16" else 1e-30       # times 1 / 6 rounds to 0 in binary16
    W = torch.zeros(3, 96, dtype=torch.float64)
    W[0, :32:2], W[0, 1:32:2] = -tiny, tiny
    W[1, 32:64:3] = -0.0
    W[2, 64:] = -1.0
    W[2, 70] = float("nan")
    W = W.to({**DT, "fp64": torch.float64}[prec]).cuda()
    codes, scales, values = lrc.q4_quantize(W, 32, torch.float16, values=True)
    c = torch.stack((codes & 15, codes >> 4), 2).view(3, -1)
    neg = torch.signbit(W)
    neg[2, 64:] = False
    assert torch.equal(c, 8 * neg.to(torch.uint8))
    assert torch.equal(torch.signbit(values[:2]), neg[:2]) and not values[:2].any() and values[2, 64:].isnan().all()
    assert not scales[:2].any() and scales[2].isnan().tolist() == [False, False, True]


@pytest.mark.parametrize("prec", ["bf16", "fp32"])
@pytest.mark.parametrize("group", [32, 64, 128, 512])
@pytest.mark.parametrize("b", [1, 20, 200])
def test_large_activations_stay_finite(lrc, prec, group, b):
    """|x| just below 2^118 at the largest weights of one sign: group sums before their scale stay in range.  All terms
    are positive: a relative error of (n + n / group + 8) 2^-24."""
    m, n = 40, 1030
    codes = torch.from_numpy(H.pack(np.full((m, n), 7))).cuda()
    scales = torch.full((m, -(-n // group)), 2.0 ** -14, dtype=torch.float16, device="cuda")
    x = 2.0 ** 118 * (1 - 2.0 ** -8)
    Y = lrc.q4_apply(codes, scales, torch.full((b, n), x, dtype=DT[prec], device="cuda"), group, out_dtype=torch.float32)
    want = n * 6 * 2.0 ** -14 * x
    assert ((Y.double() / want - 1).abs() <= (n + n / group + 8) * 2.0 ** -24).all()


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("b", [1, 8, 20, 300])
def test_small_activations_and_factors_keep_their_bits(lrc, prec, b):
    """Subnormal binary16 activations and factors, and small bfloat16 and binary32 activations: products are exact,
    so errors stay those of the sums.  Sums of one sign: relative errors of (n + n / group + 8) 2^-24 from the weights,
    (n + k + 8) 2^-24 from the compensation."""
    rng = np.random.default_rng(b)
    m, n, k, u = 70, 390, 18, 2.0 ** -24
    low = {"fp16": 2.0 ** -24, "bf16": 2.0 ** -100, "fp32": 2.0 ** -90}[prec]
    codes = rng.integers(1, 8, (m, n))
    packed = torch.from_numpy(H.pack(codes)).cuda()
    X = torch.from_numpy(low * rng.integers(1, 200, (b, n))).to(DT[prec]).cuda()
    x = X.double().cpu().numpy()
    for sprec in ("fp16", "fp32"):
        scales = torch.from_numpy(2.0 ** -24 * rng.integers(1, 900, (m, -(-n // 32)))).to(DT[sprec])
        W = H.weights(codes, scales.double().numpy(), 32)
        Y = lrc.q4_apply(packed, (scales * 2 ** 10).cuda(), X, 32, out_dtype=torch.float32)
        want = (x @ W.T) * 2.0 ** 10
        assert (abs(Y.double().cpu().numpy() - want) <= (n + n / 32 + 8) * u * want + 2.0 ** -149).all()
    zero = torch.zeros(m, -(-n // 32), dtype=torch.float32, device="cuda")
    for fprec in ("fp16", "bf16", "fp32"):
        small = 2.0 ** -24 if fprec == "fp16" else 2.0 ** -30
        U, V = (torch.from_numpy(small * rng.integers(1, 250, s)).to(DT[fprec]) for s in ((m, k), (n, k)))
        s = torch.full((k,), 2.0 ** 15, dtype=DT[fprec])
        Y = lrc.q4_apply(packed, zero, X, 32, (U.cuda(), s.cuda(), V.cuda()), out_dtype=torch.float32)
        want = ((x @ V.double().numpy()) * s.double().numpy()) @ U.double().numpy().T
        tiny = 2.0 ** -126 * k                           # results below binary32's normal range are not held to it
        assert (abs(Y.double().cpu().numpy() - want) <= (2 * n + 2 * k + 16) * u * want + tiny).all(), (fprec, sprec)
