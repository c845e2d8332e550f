"""The norm's gradient written over dy or over dsum: bit for bit what it is in a place of its own.

Sizes (in vectors of 16 bytes) at which a row's last vector is loaded by one wave alone, by threads of its own wave, and by
whole waves that own no other vector of the row (129, 130, 193), two and four vectors a thread."""
import pytest

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
@pytest.mark.parametrize("vectors", [1, 63, 64, 65, 127, 129, 130, 193, 257, 1025, 2047, 2049, 2305, 4095])
@pytest.mark.parametrize("odd", [0, 3])
def test_in_place_of_dy_and_of_dsum(lrc, prec, vectors, odd):
    n, rows = vectors * (4 if prec == "fp32" else 8) + odd, 1100
    g = torch.Generator(device="cuda").manual_seed(n)
    h, dy, ds = (torch.randn(rows, n, generator=g, device="cuda").to(DT[prec]) for _ in range(3))
    w = 1 + 0.2 * torch.randn(n, generator=g, device="cuda")
    rstd = lrc.rms_norm(h, w, stats=True)[2]
    dx, dw = lrc.rms_norm_backward(dy, h, w, rstd, dsum=ds)
    for _ in range(3):
        for mine in (dy.clone(), ds.clone()):
            over_dy = torch.equal(mine, dy)
            got = lrc.rms_norm_backward(mine if over_dy else dy, h, w, rstd, dsum=ds if over_dy else mine, dx=mine)
            assert got[0] is mine and torch.equal(mine, dx) and torch.equal(got[1], dw)
