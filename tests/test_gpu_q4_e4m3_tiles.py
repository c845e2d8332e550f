"""The 4-bit product of 8-bit activations where its results are bfloat16: the tiles on the 8-bit matrix instruction, of
every size, with every type of scales and factors.  (FP16 and FP32 results, beside them here, take the binary16 tiles.)

What the instruction does with a product of 128 columns was found by calls whose exact answers are known
(test_what_the_instruction_cuts): of each eight consecutive columns, the products are cut towards 0 to multiples of 2^-13 of
the power of two below the largest of them, and the sums of eight are added in binary32.  So a row's error is at most
seven times 2^-13 of the largest product of each eight columns, times their scale, and nothing where the activations of
each eight lie within eight binades: significands of 4 and 2 bits leave a product's last bit 4 below its exponents' sum (3 and 1),
weights span 3 binades (0.5 to 6), and 7 + 2 + 4 = 13."""
import numpy as np
import pytest

from oracle import head as H
from oracle import step as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def host(t):
    return t.double().cpu().numpy()


def half_step(prec):
    return torch.finfo(DT[prec]).eps / 2


def cut_of(X, W, rows=16):
    """(b x m) 7 2^-13 of the largest product of each eight columns, summed: X b x n and W m x n, scales included."""
    b, n = X.shape
    pad = -n % 8
    x = np.pad(np.abs(X), ((0, 0), (0, pad))).reshape(b, -1, 8)
    w = np.pad(np.abs(W), ((0, 0), (0, pad))).reshape(W.shape[0], -1, 8)
    out = np.zeros((b, W.shape[0]))
    for r in range(0, b, rows):
        for g in range(x.shape[1]):
            out[r:r + rows] += (x[r:r + rows, None, g] * w[None, :, g]).max(2)
    return 7 * 2.0 ** -13 * out


def check(got, W, X, t, factors, prec, cut):
    """got (b x m) against binary64: one rounding to its type (and the row's factor's), n sums in binary32 that the
    instruction may cut instead of rounding (two steps of 2^-24 each), the factors' part twice (its first product's sums as
    well), T' in 22 bits, and, with `cut`, what eight columns lose."""
    Xd, td = host(X.float()), host(t)[:, None]
    Y = td * H.q4_apply(W, Xd, *([] if factors is None else [host(f) for f in factors]))
    n = Xd.shape[1]
    size = np.abs(Xd) @ np.abs(W).T
    if factors is not None:
        Uf, s, V = (np.abs(host(f)) for f in factors)
        size += 2 * ((np.abs(Xd) @ V) * s) @ Uf.T
    bound = (half_step(prec) + 2 * U) * np.abs(Y) + 2 * (n + 140) * U * td * size + torch.finfo(DT[prec]).smallest_normal * half_step(prec)
    if cut:
        bound += td * cut_of(Xd, W)
    off = np.abs(host(got) - Y)
    assert np.all(off <= bound), float((off / bound).max())


def activations(g, b, n, wide):
    """e4m3 values of every binade, or 0 and the eight binades from 2 to 448."""
    x = (torch.randn(b, n, generator=g, device="cuda") * 50 * torch.exp2(-6 * torch.rand(b, n, generator=g, device="cuda"))).clamp(-448, 448)
    if not wide:
        x = torch.where(x.abs() < 2, torch.zeros_like(x), x)
    return x.to(E4M3)


def problem(seed, b, m, n, k, group, sdt, fdt, wide):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + n)
    nib = torch.randint(0, 16, (m, -(-n // 32) * 32), dtype=torch.uint8, device="cuda", generator=g)
    nib[:, n:] = 0
    scales = (torch.rand(m, -(-n // group), generator=g, device="cuda") * 0.04 + 0.01).to(DT[sdt])
    t = torch.rand(b, generator=g, device="cuda") * 0.01 + 1e-4
    F = tuple((torch.randn(*s, generator=g, device="cuda") * n ** -0.5).to(DT[fdt]) for s in ((m, k), (k,), (n, k))) if k else None
    return nib, nib[:, 0::2] | (nib[:, 1::2] << 4), scales, activations(g, b, n, wide), t, F


def some(rng, count, edges):
    return np.unique(np.concatenate([rng.integers(0, count, 40), [e for e in edges if e < count], [count - 1]]))


def weights(nib, scales, n, group, cols):
    return H.weights(nib[:, :n].cpu().numpy()[cols].astype(int), scales.double().cpu().numpy()[cols], group)


# m, n, k, group, batch: tiles of 256 x 256 (groups of 128 and more; one and odd numbers of groups a row), of 256 x 128 (groups of
# 128 in one round of them, and in two where 256 x 256 tiles take two as well; groups of 32 and 64), of 128 x 128, of 64, 32 and
# 16 rows of X, and split over columns; last tiles of a few rows and columns
SIZES = [(4100, 640, 65, 128, 4097), (8192, 130, 9, 256, 2000), (4352, 1000, 12, 512, 3850), (8200, 300, 21, 128, 1030),
         (8150, 300, 21, 128, 1010), (33000, 130, 8, 128, 300),
         (8192, 200, 33, 32, 1100), (8200, 330, 8, 64, 1030), (300, 515, 65, 128, 130), (200, 1030, 7, 32, 257), (530, 777, 20, 64, 140),
         (500, 2048, 65, 128, 64), (257, 1000, 16, 32, 50), (135, 640, 130, 64, 33), (300, 1100, 5, 256, 17), (260, 2100, 40, 32, 9)]
TYPES = [("fp16", "fp16"), ("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "fp16"), ("bf16", "fp32")]


@pytest.mark.parametrize("sdt,fdt", TYPES)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_results_of_16_bits(lrc, size, wide, sdt, fdt):
    m, n, k, group, b = size
    nib, codes, scales, X, t, F = problem(1, b, m, n, k, group, sdt, fdt, wide)
    rng = np.random.default_rng([m, n, b])
    rows, cols = some(rng, b, (0, 15, 16, 31, 63, 64, 127, 128, 255, 256)), some(rng, m, (0, 15, 63, 64, 127, 128, 255, 256))
    ri, ci = torch.from_numpy(rows).cuda(), torch.from_numpy(cols).cuda()
    W = weights(nib, scales, n, group, cols)
    Xs = X.view(torch.uint8)[ri].view(E4M3)
    whole = lrc.q4_apply(codes, scales, X, group, F, out_dtype=torch.float32, x_scales=t)
    for f in [F, None] if sdt == "fp32" else [F]:
        Fs = None if f is None else (f[0][ci], f[1], f[2])
        for prec in ("bf16", "fp32"):
            got = lrc.q4_apply(codes, scales, X, group, f, out_dtype=DT[prec], x_scales=t)
            assert torch.equal(got, lrc.q4_apply(codes, scales, X, group, f, out_dtype=DT[prec], x_scales=t))
            check(got[ri][:, ci], W, Xs, t[ri], Fs, prec, wide and prec != "fp32")
            if f is not None and prec != "fp32" and not wide:
                # all values against the ones in FP32, which other kernels compute (products of magnitudes in FP32 for the bound)
                lut = torch.from_numpy(H.E2M1).float().cuda()
                Wa = lut[(nib[:, :n] & 7).long()] * scales.float().repeat_interleave(group, dim=1)[:, :n]
                size_ = X.float().abs() @ Wa.T
                size_ += 2 * ((X.float().abs() @ F[2].float().abs()) * F[1].float().abs()) @ F[0].float().abs().T
                bound = (half_step(prec) * 1.01) * whole.abs() + 4 * (n + 140) * U * t[:, None] * size_ + 1e-37
                assert ((got.float() - whole).abs() <= bound).all()


@pytest.mark.parametrize("sdt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("fdt", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("b", [3, 20, 140])
def test_places_of_16_bits(lrc, sdt, fdt, b):
    """Rows of a larger pitch that begin off 16 bytes, in X and in Y."""
    m, n, k, group = 200, 300, 19, 64
    nib, codes, scales, X, t, F = problem(2, b, m, n, k, group, sdt, fdt, False)
    W = weights(nib, scales, n, group, np.arange(m))
    big = torch.full((b, n + 5), 0x7F, dtype=torch.uint8, device="cuda").view(E4M3)
    big.view(torch.uint8)[:, 1:1 + n] = X.view(torch.uint8)
    for prec in ("bf16", "fp16"):
        Y = torch.full((b, 210), 7.0, dtype=DT[prec], device="cuda")
        got = lrc.q4_apply(codes, scales, big[:, 1:1 + n], group, F, Y=Y[:, 3:203], x_scales=t)
        check(got, W, X, t, F, prec, False)
        assert (Y[:, :3] == 7).all() and (Y[:, 203:] == 7).all()
        assert torch.equal(got, lrc.q4_apply(codes, scales, X, group, F, out_dtype=DT[prec], x_scales=t))


@pytest.mark.parametrize("b", [12, 40, 200])
@pytest.mark.parametrize("prec", ["bf16", "fp16"])
def test_every_code(lrc, b, prec):
    """All 256 codes of activations, one a result: 16 bits hold each."""
    m, n = 256, 256
    one = torch.zeros(m, n // 2, dtype=torch.uint8, device="cuda")
    i = torch.arange(m, device="cuda")
    one[i, i // 2] = torch.where(i % 2 == 1, 0x20, 0x02).to(torch.uint8)              # row i takes column i, with weight 1
    scales = torch.ones(m, 2, dtype=torch.float16, device="cuda")
    X = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(b, 1)
    X[:, [0x7F, 0xFF]] = 0
    X = torch.stack([x.roll(7 * r) for r, x in enumerate(X)]).view(E4M3)
    got = lrc.q4_apply(one, scales, X, 128, out_dtype=DT[prec], x_scales=torch.ones(b, device="cuda"))
    assert torch.equal(got.float(), X.float())


@pytest.mark.parametrize("m,n,group,b", [(8192, 300, 128, 2048), (8192, 200, 64, 1100), (300, 520, 32, 140), (200, 300, 128, 40), (100, 640, 256, 12)])
def test_what_is_not_finite_stays_in_its_row_and_column(lrc, m, n, group, b):
    nib, codes, scales, X, t, F = problem(3, b, m, n, 8, group, "fp32", "fp16", True)
    want = lrc.q4_apply(codes, scales, X, group, F, x_scales=t)
    assert want.dtype == torch.bfloat16 and torch.isfinite(want).all()
    rows, cols = torch.ones(b, dtype=torch.bool, device="cuda"), torch.ones(m, dtype=torch.bool, device="cuda")
    X.view(torch.uint8)[b // 3, n - 1] = 0x7F
    X.view(torch.uint8)[0, 0] = 0xFF
    t[b - 1] = float("nan")
    scales[m - 1, -1] = float("nan")
    scales[m // 2, 0] = float("inf")
    for r in (b // 3, 0, b - 1):
        rows[r] = False
    cols[m - 1] = cols[m // 2] = False
    got = lrc.q4_apply(codes, scales, X, group, F, x_scales=t)
    assert torch.isnan(got[~rows]).all() and torch.isnan(got[:, m - 1]).all() and not torch.isfinite(got[:, m // 2]).any()
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])


def test_what_the_instruction_cuts(lrc):
    """Large products that cancel beside a small one, in the same eight columns and outside of them: the rule above, and no
    more than it."""
    b, m, n = 16, 16, 128

    def call(w, x, dt=torch.bfloat16):
        nib, X = np.zeros((m, n), int), torch.zeros(b, n)
        for c, v in w:
            nib[:, c] = list(H.E2M1).index(abs(v)) + 8 * (v < 0)
        for c, v in x:
            X[:, c] = v
        y = lrc.q4_apply(torch.from_numpy(H.pack(nib)).cuda(), torch.ones(m, 1, device="cuda"), X.to(E4M3).cuda(), 128, out_dtype=dt,
                         x_scales=torch.ones(b, device="cuda"))
        assert (y == y[0, 0]).all()
        return float(y[0, 0])

    for at, big in ((0, 256.0), (40, 448.0), (120, 8.0)):
        for e in range(-10, 6):
            small = 2.0 ** e
            if small * 2 > 448 or small * 2 < 2.0 ** -9:
                continue
            w, x = [(at, 4), (at + 1, -4)], [(at, big), (at + 1, big)]
            inside = call(w + [(at + 5, 0.5)], x + [(at + 5, 2 * small)])
            unit = 2.0 ** -13 * 4 * 2.0 ** np.floor(np.log2(big))
            assert inside == np.floor(small / unit) * unit
            assert call(w + [((at + 8) % n, 0.5)], x + [((at + 8) % n, 2 * small)]) == small
            assert call(w + [(at + 5, -0.5)], x + [(at + 5, 2 * small)]) == -inside
            assert call(w + [(at + 5, 0.5)], x + [(at + 5, 2 * small)], torch.float32) == small
