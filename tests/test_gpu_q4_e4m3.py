"""The 4-bit product of 8-bit activations against the binary64 oracle.

Tolerances: products are exact, sums of n products in binary32 are within n * 2^-24 of the sum of magnitudes, and the
result is rounded once (after the row's factor, one rounding more)."""
import numpy as np
import pytest

from oracle import head as H
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


def host(t):
    return t.double().cpu().numpy()


def problem(seed, b, m, n, k, group, sdt="fp16", fdt="fp16", pad=0):
    rng = np.random.default_rng([seed, b, m, n, k, group])
    codes = rng.integers(0, 16, (m, n))
    scales = torch.from_numpy(rng.uniform(0.01, 0.05, (m, -(-n // group)))).to(DT[sdt])
    W = H.weights(codes, scales.double().numpy(), group)
    X = torch.from_numpy(O.e4m3_nearest(rng.normal(size=(b, n)) * 100)).float().to(torch.float8_e4m3fn)
    t = torch.from_numpy(rng.uniform(0.001, 0.01, b).astype(np.float32))
    factors = None
    if k:
        factors = tuple(torch.from_numpy(rng.normal(size=s) * n ** -0.5).to(DT[fdt]).cuda() for s in ((m, k), (k,), (n, k)))
    x = X.cuda()
    if pad:
        big = torch.zeros(b, n + pad, dtype=torch.uint8, device="cuda").fill_(0x7F).view(torch.float8_e4m3fn)     # NaN around
        x = big[:, 1:1 + n]
        x.copy_(X.cuda())
    return torch.from_numpy(H.pack(codes)).cuda(), scales.cuda(), x, t.cuda(), factors, W


def check(got, W, X, t, factors, prec):
    Xd, td = host(X.float()), host(t)[:, None]
    Y = td * H.q4_apply(W, Xd, *([] if factors is None else [host(f) for f in factors]))
    n = Xd.shape[1]
    size = np.abs(Xd) @ np.abs(W).T
    if factors is not None:
        Uf, s, V = (np.abs(host(f)) for f in factors)
        size += 2 * ((np.abs(Xd) @ V) * s) @ Uf.T
    bound = (torch.finfo(DT[prec]).eps / 2 + 2 * U) * np.abs(Y) + (n + 140) * U * td * size + \
        torch.finfo(DT[prec]).smallest_normal * torch.finfo(DT[prec]).eps / 2
    off = np.abs(host(got) - Y)
    assert np.all(off <= bound), float((off / bound).max())


SIZES = [(1, 1, 1, 0, 32), (1, 48, 200, 7, 32), (2, 17, 33, 0, 64), (7, 300, 1000, 65, 128), (8, 530, 513, 5, 32), (9, 130, 260, 12, 64),
         (16, 257, 129, 0, 128), (17, 64, 2048, 33, 256), (33, 400, 640, 65, 512), (48, 512, 384, 16, 128), (64, 129, 1027, 40, 64),
         (65, 300, 700, 20, 32), (130, 513, 515, 65, 128), (257, 260, 1030, 9, 64), (300, 1100, 256, 0, 128)]


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_product(lrc, prec, size):
    b, m, n, k, group = size
    codes, scales, X, t, factors, W = problem(1, *size, pad=0 if b % 2 else 3)
    got = lrc.q4_apply(codes, scales, X, group, factors, out_dtype=DT[prec], x_scales=t)
    assert got.dtype == DT[prec]
    check(got, W, X, t, factors, prec)
    assert torch.equal(got, lrc.q4_apply(codes, scales, X, group, factors, out_dtype=DT[prec], x_scales=t))


@pytest.mark.parametrize("sdt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("fdt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("b", [3, 20, 140])
def test_types_of_scales_and_factors(lrc, sdt, fdt, b):
    codes, scales, X, t, factors, W = problem(2, b, 200, 300, 19, 64, sdt, fdt)
    Y = torch.full((b, 210), 7.0, dtype=torch.float32, device="cuda")
    got = lrc.q4_apply(codes, scales, X, 64, factors, Y=Y[:, 4:204], x_scales=t)
    check(got, W, X, t, factors, "fp32")
    assert (Y[:, :4] == 7).all() and (Y[:, 204:] == 7).all()


@pytest.mark.parametrize("b", [1, 12, 200])
def test_every_code_and_what_is_not_finite(lrc, b):
    """All 256 activations codes of a row against unit weights; NaN codes and factors reach their row alone."""
    m, n = 40, 256
    codes = torch.full((m, 128), 0x22, dtype=torch.uint8, device="cuda")              # weights of 1
    codes[1] = 0xAA                                                                   # of -1
    scales = torch.ones(m, 2, dtype=torch.float16, device="cuda")
    all_codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    X = torch.zeros(b, n, dtype=torch.uint8, device="cuda")
    X[-1] = all_codes
    X[-1][[0x7F, 0xFF]] = 0
    t = torch.ones(b, device="cuda")
    eye = torch.zeros(n, 32, dtype=torch.uint8, device="cuda")
    got = lrc.q4_apply(codes, scales, X.view(torch.float8_e4m3fn), 128, out_dtype=torch.float32, x_scales=t)
    assert got[-1].abs().max() == 0                                                   # the signs cancel
    one = torch.zeros(m, 128, dtype=torch.uint8, device="cuda")
    for i in range(m):
        one[i, (6 * i + 1) // 2] = 0x20 if (6 * i + 1) % 2 else 0x02                   # row i takes column 6 i + 1
    got = lrc.q4_apply(one, scales, X.view(torch.float8_e4m3fn), 128, out_dtype=torch.float32, x_scales=t)
    want = X.view(torch.float8_e4m3fn).float()[:, 1:6 * m:6][:, :m]
    assert torch.equal(got, want)
    del eye
    X[0, 5] = 0x7F
    got = lrc.q4_apply(codes, scales, X.view(torch.float8_e4m3fn), 128, out_dtype=torch.float32, x_scales=t)
    assert torch.isnan(got[0]).all() and torch.isfinite(got[1:]).all()
    t[-1] = float("nan")
    got = lrc.q4_apply(codes, scales, X.view(torch.float8_e4m3fn), 128, x_scales=t)
    assert got.dtype == torch.bfloat16 and torch.isnan(got[-1]).all()


@pytest.mark.parametrize("m,n,k,group,b", [(4100, 640, 65, 128, 4097), (8192, 130, 0, 256, 2000), (4352, 1000, 9, 512, 3850)])
@pytest.mark.parametrize("sdt", ["fp32", "fp16", "bf16"])
def test_large_tiles(lrc, m, n, k, group, b, sdt):
    """Products of a tile for every compute unit: sampled rows and columns, and the rest against them twice."""
    rng = np.random.default_rng([m, n, b])
    codes = torch.randint(0, 256, (m, (n + 31) // 32 * 16), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(n))
    nib = torch.stack((codes & 15, codes >> 4), 2).view(m, -1)
    nib[:, n:] = 0
    codes = nib[:, 0::2] | (nib[:, 1::2] << 4)
    scales = (torch.rand(m, -(-n // group), device="cuda") * 0.04 + 0.01).to(DT[sdt])
    X = (torch.randn(b, n, device="cuda") * 50).clamp(-440, 440).to(torch.float8_e4m3fn)
    t = torch.rand(b, device="cuda") * 0.01
    F = tuple((torch.randn(*s, device="cuda") * n ** -0.5).half() for s in ((m, k), (k,), (n, k))) if k else None
    got = lrc.q4_apply(codes, scales, X, group, F, out_dtype=torch.float32, x_scales=t)
    rows = np.unique(np.concatenate([rng.integers(0, b, 60), [0, 255, 256, b - 1]]))
    cols = np.unique(np.concatenate([rng.integers(0, m, 60), [0, 63, 64, 255, 256, m - 1]]))
    W = H.weights(nib[:, :n].cpu().numpy()[cols].astype(int), scales.double().cpu().numpy()[cols], group)
    Fs = None if F is None else (F[0][torch.from_numpy(cols).cuda()], F[1], F[2])
    ri = torch.from_numpy(rows).cuda()
    check(got[ri][:, torch.from_numpy(cols).cuda()], W, X.view(torch.uint8)[ri].view(torch.float8_e4m3fn), t[ri], Fs, "fp32")
    # every other value: halves of the batch, which take other tiles
    for part in (slice(0, b // 8), slice(b // 8, b // 3)):
        small = lrc.q4_apply(codes, scales, X[part], group, F, out_dtype=torch.float32, x_scales=t[part])
        size = got[part].abs().mean()
        assert (small - got[part]).abs().max() <= 1e-4 * size * 10


@pytest.mark.parametrize("b", [1, 8, 9, 17, 48, 64, 65, 130, 300])
@pytest.mark.parametrize("m,n,group", [(300, 1024, 128), (2100, 1000, 32), (530, 777, 64), (260, 1024, 512)])
def test_sums_hold_32_bits(lrc, b, m, n, group):
    """Whole activations and weights whose sums stay below 2^24 (1024 * 448 * 12 = 5.5e6): every partial sum is a whole number
    that binary32 holds, so a result in FP32 is exact, whatever the order of its sums."""
    rng = np.random.default_rng([5, b, m, n])
    codes, scales = rng.integers(0, 16, (m, n)), torch.full((m, -(-n // group)), 2.0).half()
    W = H.weights(codes, scales.double().numpy(), group)
    whole = O.E4M3[(O.E4M3 == np.floor(O.E4M3))]
    X = torch.from_numpy(rng.choice(whole, (b, n)) * rng.choice([-1.0, 1.0], (b, n))).float().to(torch.float8_e4m3fn).cuda()
    t = torch.from_numpy(2.0 ** rng.integers(-3, 4, b)).float().cuda()
    want = host(t)[:, None] * (host(X.float()) @ W.T)
    got = lrc.q4_apply(torch.from_numpy(H.pack(codes)).cuda(), scales.cuda(), X, group, out_dtype=torch.float32, x_scales=t)
    assert np.array_equal(host(got), want)
