"""A workgroup a row at a vocabulary below the split's, rows of every kind, against the binary64 oracle: u lies in the
middle of a kept token's interval of at least 1e-4 of the mass, so that rounding does not decide."""
import numpy as np
import pytest

from oracle import head as H
from test_gpu_sample_split import rows_of_every_kind

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("prec", [torch.float32, torch.float16, torch.bfloat16])
def test_rows_of_every_kind(lrc, prec):
    V = 20011
    g = torch.Generator(device="cuda").manual_seed(V)
    L = rows_of_every_kind(g, V, {torch.float32: "fp32", torch.float16: "fp16", torch.bfloat16: "bf16"}[prec])
    host = L.double().cpu().numpy()
    rng = np.random.default_rng(V)
    n = len(host)
    for k in (0, 1, 7, 300):
        for T in (0.3, 1.0):
            u, want = np.full(n, 0.5), np.full(n, -1)
            for r in range(2, n):
                l = np.where(np.isnan(host[r]), -np.inf, host[r])
                if np.isposinf(l).any():
                    want[r] = l.argmax()
                    continue
                _, kept = H.sample_kept(l, T, k)
                c = kept / kept.sum()
                wide = np.flatnonzero(c >= (1e-4 if (c >= 1e-4).any() else c.max()))
                j = int(rng.choice(wide))
                u[r], want[r] = c[:j].sum() + c[j] / 2, j
            f = lambda x: torch.tensor(np.asarray(x, np.float32), device="cuda")  # noqa: E731
            got = lrc.sample(L, f(u), f(np.full(n, T)), torch.full((n,), k, device="cuda"))
            ok = (got.cpu().numpy() == want)
            # an even row of 20011 tokens: u in binary32 resolves a token's interval, the sum's last bits may not
            assert ok.all(), (k, T, np.flatnonzero(~ok), got.cpu().numpy()[~ok], want[~ok])
