"""4-bit products at the sizes where the planner changes kernels and where a kernel changes buffers, against binary64.

Tolerance: with u = 2^-24, (n + n / group + 8) u (|X| |W|^T) for the sums and (n + k + 8) u (|X| |V| |s| |U|^T) for the
compensation; outputs are stored in binary32 (half an ulp, 2^-24 |Y|)."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
E2M1 = [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def product(lrc, seed, m, n, b, group, prec, sprec, k, fprec="fp16"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 16, (m, n), generator=g, device="cuda")
    full = torch.zeros(m, -(-n // 32) * 32, dtype=torch.uint8, device="cuda")
    full[:, :n] = codes
    packed = full[:, 0::2] | (full[:, 1::2] << 4)
    scales = (0.0125 + 0.05 * torch.rand(m, -(-n // group), generator=g, device="cuda")).to(DT[sprec])
    X = torch.randn(b, n, generator=g, device="cuda").to(DT[prec])
    F = tuple((torch.randn(*s, generator=g, device="cuda") * c).to(DT[fprec]) for s, c in
              (((m, k), m ** -0.5), ((k,), 1.0), ((n, k), n ** -0.5))) if k else None
    Y = lrc.q4_apply(packed, scales, X, group, F, out_dtype=torch.float32)
    u, x = 2.0 ** -24, X.double()
    W = torch.tensor(E2M1, dtype=torch.float64, device="cuda")[codes]
    W *= scales.double().repeat_interleave(group, 1)[:, :n]
    ref = x @ W.t().contiguous()
    bound = (n + n / group + 8) * u * (x.abs() @ W.abs().t().contiguous())
    if k:
        U, s, V = (f.double() for f in F)
        ref += ((x @ V) * s) @ U.t().contiguous()
        bound += (n + k + 8) * u * (((x.abs() @ V.abs()) * s.abs()) @ U.abs().t().contiguous())
    err = (Y.double() - ref).abs()
    assert (err <= bound + u * ref.abs()).all(), float((err / bound).max())
    assert err.norm() <= 1e-5 * ref.norm()
    assert torch.equal(Y, lrc.q4_apply(packed, scales, X, group, F, out_dtype=torch.float32))


@pytest.mark.parametrize("prec", ["fp16", "bf16"])
@pytest.mark.parametrize("sprec", ["fp16", "fp32"])
@pytest.mark.parametrize("group", [32, 64, 128, 512])
@pytest.mark.parametrize("m,n,b,k", [(4001, 640, 2005, 0), (3841, 300, 1921, 21), (7937, 1184, 1025, 5)])
def test_prompt_tiles(lrc, prec, sprec, group, m, n, b, k):
    """ceil(m / 256) ceil(b / 128) >= 256: the largest tiles, over their ends along W and X, packed and in place."""
    assert -(-m // 256) * -(-b // 128) >= 256
    product(lrc, m + group, m, n, b, group, prec, sprec, k)


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [100, 9000, 16400])
@pytest.mark.parametrize("b", [1, 2, 5, 8])
def test_few_rows_longer_than_one_chunk(lrc, prec, group, m, b):
    """More columns than the row kernel holds in LDS at a time (2048 to 8192), for one and two row blocks a wave and for
    four and eight waves."""
    for n in (8193, 12365):
        product(lrc, m + b, m, n, b, group, prec, "bf16" if b == 2 else "fp16", 9 if b < 5 else 0)


@pytest.mark.parametrize("prec", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("b", [7, 8, 9, 16, 17, 32, 33, 64, 65, 128])
def test_every_number_of_rows_around_a_change_of_kernel(lrc, prec, b):
    for group in (32, 128):
        product(lrc, b, 1030, 1000, b, group, prec, "fp32", 17, "bf16")
