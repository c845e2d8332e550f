"""4-bit quantization and product against the binary64 oracle (oracle/head.py).

Tolerances.  Codes, scales and values follow a definition in IEEE operations and are compared exactly.  The product's
sums hold at most n exact products and n / group scaled partial sums, then k + 1 terms of the compensation, each formed
from a sum of n terms: with u = 2^-24 the error of an output is at most (n + n / group + 8) u (|X| |W|^T) +
(n + k + 8) u (|X| |V| |s| |U|^T), then half an ulp of the stored type.  The relative Frobenius error is held to the
framework's bounds of the stored type (binary32 1e-5, binary16 2e-3; bfloat16 has 3 bits less, 16e-3)."""
import numpy as np
import pytest

from oracle import head as H

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp64": torch.float64, "fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -24, "bf16": 2.0 ** -133}
FRO = {"fp32": 1e-5, "fp16": 2e-3, "bf16": 16e-3}


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def up(x):
    return x.double().cpu().numpy()


def stored(rng, shape, prec, scale=1.0):
    return torch.from_numpy(rng.normal(size=shape) * scale).to(DT[prec]).cuda()


def head(rng, m, n, group, sprec="fp16", scale=0.05):
    codes = rng.integers(0, 16, (m, n))
    scales = torch.from_numpy(scale * (0.25 + rng.random((m, -(-n // group))))).to(DT[sprec])
    return H.weights(codes, up(scales), group), torch.from_numpy(H.pack(codes)).cuda(), scales.cuda()


def check(Y, W, X, yprec, group, factors=None):
    got, X = up(Y), up(X)
    m, n = W.shape
    u = 2.0 ** -24
    if factors is None:
        ref, bound = H.q4_apply(W, X), (n + n / group + 8) * u * (abs(X) @ abs(W).T)
    else:
        U, s, V = (up(f) for f in factors)
        ref = H.q4_apply(W, X, U, s, V)
        bound = ((n + n / group + 8) * u * (abs(X) @ abs(W).T)
                 + (n + len(s) + 8) * u * ((abs(X) @ abs(V)) * abs(s)) @ abs(U).T)
    bound = bound + UNIT[yprec] * abs(ref) + TINY[yprec]
    assert got.shape == ref.shape
    assert (abs(got - ref) <= bound).all(), float((abs(got - ref) / bound).max())
    assert np.linalg.norm(got - ref) <= FRO[yprec] * np.linalg.norm(ref)


# ------------------------------------------------------------------ quantize --

@pytest.mark.parametrize("prec", ["fp64", "fp32", "fp16", "bf16"])
@pytest.mark.parametrize("m,n,group", [(1, 1, 32), (3, 31, 32), (2, 512, 512), (5, 33, 64), (7, 1000, 128), (130, 513, 256),
                                       (9, 4099, 32)])
def test_quantize_matches_oracle(lrc, prec, m, n, group):
    rng = np.random.default_rng(100 + n)
    W = stored(rng, (m, n), prec, 0.02)
    W[:, ::5] = 0
    for sprec in ("fp16", "fp32", "bf16"):
        codes, scales, values = lrc.q4_quantize(W, group, DT[sprec], values=True)
        host = W.cpu() if prec == "fp64" else W.float().cpu()
        cast = lambda x: torch.from_numpy(x).to(DT[sprec]).double().numpy()  # noqa: E731
        c, s = H.quantize(host.numpy(), group, cast, np.float64 if prec == "fp64" else np.float32)
        assert np.array_equal(up(scales), s)
        assert np.array_equal(codes.cpu().numpy(), H.pack(c))
        want = torch.from_numpy(H.weights(c, s, group)).to(DT["fp32"] if prec != "fp64" else DT["fp64"]).to(DT[prec])
        assert torch.equal(values.cpu(), want)
        assert not codes.cpu().numpy()[:, (n + 1) // 2:].any()


def test_quantize_pitch_and_alignment(lrc):
    rng = np.random.default_rng(5)
    big = stored(rng, (40, 331), "fp32")
    for W in (big[:, :300], big[:, 1:290], big[3:, 2:3], big.t()[:300].t()):
        if W.stride(1) != 1 and W.shape[1] > 1:
            with pytest.raises(ValueError, match="contiguous"):
                lrc.q4_quantize(W, 32)
            continue
        a = lrc.q4_quantize(W, 32, values=True)
        b = lrc.q4_quantize(W.contiguous(), 32, values=True)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_quantize_zero_tiny_and_non_finite_groups(lrc):
    W = torch.zeros(6, 96, device="cuda")
    W[0, :32] = 1e-30                   # the binary16 scale is 0
    W[1, 40] = float("nan")
    W[2, 70] = float("-inf")
    W[3, 5] = 1e6                       # the binary16 scale overflows
    W[4] = -0.0
    W[5, 1] = -3.0
    codes, scales, values, bad = lrc.q4_quantize(W, 32, values=True, count_nonfinite=True)
    assert bad == 3
    s = up(scales)
    assert np.isnan(s[1, 1]) and np.isnan(s[2, 2]) and np.isnan(s[3, 0])
    assert np.isnan(up(values)[1, 32:64]).all() and np.isfinite(up(values)[1, :32]).all()
    assert s[0, 0] == 0 and not values[0].any() and not codes[0].any()
    assert float(values[5, 1]) == -3.0 and torch.signbit(values[4]).all()
    assert lrc.q4_quantize(W, 32, torch.float32, count_nonfinite=True)[2] == 2


# ------------------------------------------------------------------- product --

@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("m,n,group,b", [(1, 1, 32, 1), (17, 33, 32, 1), (16, 128, 128, 1), (100, 500, 64, 3),
                                         (65, 1025, 128, 16), (257, 2049, 32, 17), (130, 640, 256, 33), (48, 4099, 512, 64),
                                         (70, 300, 64, 65), (300, 260, 128, 130), (640, 384, 32, 257)])
def test_product_matches_oracle(lrc, prec, m, n, group, b):
    rng = np.random.default_rng(m * 1000 + n + b)
    W, codes, scales = head(rng, m, n, group)
    X = stored(rng, (b, n), prec)
    check(lrc.q4_apply(codes, scales, X, group), W, X, prec, group)
    for k in {1, min(21, m, n), min(m, n, 130)}:
        for fprec in ("fp16", "fp32", "bf16"):
            F = (stored(rng, (m, k), fprec, m ** -0.5), stored(rng, (k,), fprec), stored(rng, (n, k), fprec, n ** -0.5))
            for yprec in {prec, "fp32"}:
                Y = lrc.q4_apply(codes, scales, X, group, F, out_dtype=DT[yprec])
                check(Y, W, X, yprec, group, F)


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("m,n,k,b", [(8192, 2048, 33, 1), (20000, 1056, 0, 5), (4111, 3000, 65, 48), (1500, 1000, 40, 700),
                                     (2048, 1024, 65, 512), (512, 8192, 64, 2)])
def test_product_at_size(lrc, prec, m, n, k, b):
    rng = np.random.default_rng(m + n + b)
    W, codes, scales = head(rng, m, n, 128, "fp32")
    X = stored(rng, (b, n), prec)
    F = None
    if k:
        F = (stored(rng, (m, k), "fp16", m ** -0.5), stored(rng, (k,), "fp16"), stored(rng, (n, k), "fp16", n ** -0.5))
    Y = lrc.q4_apply(codes, scales, X, 128, F, out_dtype=torch.float32)
    check(Y, W, X, "fp32", 128, F)
    assert torch.equal(Y, lrc.q4_apply(codes, scales, X, 128, F, out_dtype=torch.float32))


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("b", [1, 20, 300])
def test_product_pitches_and_misaligned_bases(lrc, prec, b):
    rng = np.random.default_rng(b)
    m, n = 150, 290
    W, codes, scales = head(rng, m, n, 32)
    base = stored(rng, (b, 310), prec)
    base.view(-1)[::310] = 3e4                      # outside the operand
    out = torch.full((b, 170), 7.0, dtype=DT[prec], device="cuda")
    X, Y = base[:, 3:3 + n], out[:, 5:5 + m]
    lrc.q4_apply(codes, scales, X, 32, Y=Y)
    check(Y, W, X, prec, 32)
    assert (out[:, :5] == 7).all() and (out[:, 5 + m:] == 7).all()


def test_product_ignores_what_lies_past_a_row(lrc):
    """NaN beyond the n activations of a row, and beyond the last row, is never read into a sum."""
    rng = np.random.default_rng(3)
    for n, b in ((100, 1), (129, 5), (33, 70)):
        W, codes, scales = head(rng, 40, n, 64)
        base = torch.full((b + 3, n + 30), float("nan"), dtype=torch.float16, device="cuda")
        base[:b, :n] = stored(rng, (b, n), "fp16")
        check(lrc.q4_apply(codes, scales, base[:b, :n], 64), W, base[:b, :n], "fp16", 64)


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("b", [2, 90])
def test_product_non_finite_activations_stay_in_their_row(lrc, prec, b):
    rng = np.random.default_rng(8)
    m, n = 33, 200
    W, codes, scales = head(rng, m, n, 32)
    X = stored(rng, (b, n), prec)
    clean = lrc.q4_apply(codes, scales, X, 32)
    Z = X.clone()
    Z[1, 7] = float("inf")
    Y = lrc.q4_apply(codes, scales, Z, 32)
    assert torch.equal(Y[0], clean[0]) and torch.equal(Y[2:], clean[2:])
    w = W[:, 7]
    got = up(Y)[1]
    assert np.isnan(got[w == 0]).all() and (got[w > 0] == np.inf).all() and (got[w < 0] == -np.inf).all()
    Z[1, 7] = float("nan")
    Y = lrc.q4_apply(codes, scales, Z, 32)
    assert Y[1].isnan().all() and torch.equal(Y[0], clean[0])


def test_product_of_binary32_keeps_its_bits(lrc):
    """Binary32 activations over the exponent range: relative errors stay at binary32 rounding, not bfloat16's."""
    rng = np.random.default_rng(9)
    codes = np.zeros((16, 64), np.int64)
    codes[np.arange(16), np.arange(16)] = 2             # one weight of 1 a row: the product copies an activation
    packed = torch.from_numpy(H.pack(codes)).cuda()
    one = torch.ones(16, 2, device="cuda")
    x = torch.from_numpy((1 + rng.random((70, 64))) * 2.0 ** rng.integers(-100, 120, (70, 64))).float().cuda()
    for b in (1, 70):
        assert torch.equal(lrc.q4_apply(packed, one, x[:b], 32), x[:b, :16])


def test_product_zero_rows_and_streams(lrc):
    rng = np.random.default_rng(4)
    W, codes, scales = head(rng, 64, 96, 32)
    assert lrc.q4_apply(codes, scales, torch.empty(0, 96, device="cuda"), 32).shape == (0, 64)
    st = torch.cuda.Stream()
    F = (stored(rng, (64, 8), "fp16"), stored(rng, (8,), "fp16"), stored(rng, (96, 8), "fp16"))
    X = stored(rng, (9, 96), "bf16")
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        Y = lrc.q4_apply(codes, scales, X, 32, F)
    st.synchronize()
    check(Y, W, X, "bf16", 32, F)
