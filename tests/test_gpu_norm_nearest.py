"""The 8-bit norm's codes are the e4m3 values nearest to the binary32 quotient y / scale, ties to even, also beside the
middles of two values.

Rows of ones without eps have the inverse root 1, so y is the weight itself, whatever binary32 value that is."""
import numpy as np
import pytest

from oracle import step as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
MIDDLES = (O.E4M3[1:] + O.E4M3[:-1]) / 2


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("n", [1765, 1768, 45000])
@pytest.mark.parametrize("amax", [448.0, 1.0, 0.7310585, 5.1e-3, 1.7e5, 3.1e38, 2.9e-17, 3.3e-36, 7.7e-41])
def test_codes_beside_the_middles(lrc, prec, n, amax):
    amax = np.float32(amax)
    t = amax / np.float32(448.0)
    assert t > 0
    w = [amax]
    for m in MIDDLES:
        near = np.float32(m * float(t))
        for step in range(-3, 4):
            y = near
            for _ in range(abs(step)):
                y = np.nextafter(y, np.float32(np.inf if step > 0 else -np.inf), dtype=np.float32)
            w += [y, -y]
    w = np.array(w, np.float32)
    w[np.abs(w) > amax] = amax
    w = np.concatenate([w, np.full(n - len(w), -0.0, np.float32)])
    w = w[np.random.default_rng(n).permutation(n)]
    x = torch.ones(3, n, dtype=DT[prec], device="cuda")
    codes, scales, _ = lrc.rms_norm_e4m3(x, torch.from_numpy(w).cuda(), eps=0.0)
    assert (scales.cpu().numpy() == t).all()
    got = codes.float().cpu().numpy()
    want = O.e4m3_nearest(w / t)                                # numpy's binary32 division
    for row in got:
        assert np.array_equal(row, want) and np.array_equal(np.signbit(row), np.signbit(want))

