"""Sampling against the binary64 oracle (oracle/head.py).

A token is a whole number, so the tests draw where rounding cannot decide: u lies in the middle of a token's interval
that is at least 1e-4 of the kept mass wide (weights are binary32 values with relative errors below 1e-5), and top-p,
min-p thresholds lie between two tokens by the same margin."""
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


def f32(x):
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


def p_between(l, T, k, rng):
    """A top-p threshold with a margin: halfway into the token that the cut keeps last."""
    order, kept = H.sample_kept(l, T, k)
    ws = kept[order]
    ws = ws[ws > 0] / ws.sum()
    wide = np.flatnonzero(ws >= 1e-4)
    if len(wide) == 0:
        return 1.0
    j = int(rng.choice(wide))
    before = ws[:j].sum()
    return float(np.float32(before + ws[j] / 2))


def u_inside(kept, rng):
    """(u, token): u in the middle of a kept token's interval."""
    c = kept / kept.sum()
    wide = np.flatnonzero(c >= 1e-4)
    j = int(rng.choice(wide))
    return float(c[:j].sum() + c[j] / 2), j


def rows_of(rng, rows, V, prec, masked=0.0, spread=2.0):
    l = rng.normal(size=(rows, V)) * spread
    for r in range(rows):
        l[r, rng.integers(0, V, min(6, V))] += 6.0     # a few likely tokens, so that intervals are wide
    if masked:
        gone = rng.random((rows, V)) < masked
        gone[np.arange(rows), rng.integers(0, V, rows)] = False
        l[gone] = -np.inf
    return torch.from_numpy(l).to(DT[prec]).cuda()


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (2, 63), (40, 257), (5, 8191), (3, 8192), (9, 32003), (2, 131071), (1, 200003)])
@pytest.mark.parametrize("masked", [0.0, 0.9])
def test_sample_matches_oracle(lrc, prec, rows, V, masked):
    rng = np.random.default_rng(rows * 7 + V)
    L = rows_of(rng, rows, V, prec, masked)
    host = L.double().cpu().numpy()
    T, K, P, MP, U, want = [], [], [], [], [], []
    for r in range(rows):
        t = float(np.float32(rng.uniform(0.5, 1.5)))
        k = int(rng.choice([0, 1, 2, 5, 40, 1000, V, V + 3]))
        p = p_between(host[r], t, k, rng) if rng.random() < 0.6 else 1.0
        mp = 0.0
        if rng.random() < 0.4:                          # between two weights
            w = np.unique(np.exp((host[r][np.isfinite(host[r])] - host[r].max()) / t))
            i = int(rng.integers(0, len(w)))
            lo = w[i - 1] if i else 0.0
            if w[i] > lo * 1.001 and w[i] > 1e-6:
                mp = float(np.float32((lo + w[i]) / 2))
        _, kept = H.sample_kept(host[r], t, k, p, mp)
        u, j = u_inside(kept, rng)
        T.append(t), K.append(k), P.append(p), MP.append(mp), U.append(u), want.append(j)
    got = lrc.sample(L, f32(U), f32(T), torch.tensor(K, device="cuda"), f32(P), f32(MP))
    assert got.cpu().tolist() == want


def test_sample_without_parameters_and_extremes_of_u(lrc):
    L = torch.tensor([[0.0, float("-inf"), 1.0, float("-inf")]] * 6, device="cuda")
    u = f32([0.0, -1.0, float("nan"), 0.999999, 1.0, 7.0])
    assert lrc.sample(L, u).cpu().tolist() == [0, 0, 0, 2, 2, 2]


def test_sample_ties_go_to_the_lowest_index(lrc):
    V = 50000
    L = torch.full((5, V), 3.0, device="cuda")
    L[:, 100] = -5.0
    k = torch.tensor([3, 3, 1, 200, 0], device="cuda")
    u = f32([0.99, 0.5, 0.9, 0.999, 0.99999])
    T = f32([1, 1, 1, 1, 0])
    # the kept are 0..k-1 without 100
    assert lrc.sample(L, u, T, k).cpu().tolist() == [2, 1, 0, 200, 0]
    p = f32([1.0, 0.5 / V, 2.5 / V, 1.0, 1.0])          # the first, then the first three
    assert lrc.sample(L, f32([0.0, 0.9, 0.9, 0.0, 0.0]), T, None, p).cpu().tolist() == [0, 0, 2, 0, 0]
    for dt in (torch.float16, torch.bfloat16):
        assert lrc.sample(L.to(dt), u, T, k).cpu().tolist() == [2, 1, 0, 200, 0]


def test_sample_greedy_and_odd_temperatures(lrc):
    rng = np.random.default_rng(2)
    L = rows_of(rng, 8, 5000, "fp32")
    best = L.double().cpu().numpy().argmax(1).tolist()
    u = f32(np.full(8, 0.7))
    for t in (0.0, -1.0, float("nan"), 1e-30, 1e-45):
        assert lrc.sample(L, u, f32([t] * 8)).cpu().tolist() == best
    # an infinite temperature draws evenly from the finite logits
    M = torch.full((1, 1000), float("-inf"), device="cuda")
    M[0, 10:20] = torch.arange(10.0, device="cuda")
    for i in range(10):
        assert lrc.sample(M, f32([(i + 0.5) / 10]), f32([float("inf")])).item() == 10 + i


def test_sample_rows_without_a_choice(lrc):
    L = torch.zeros(6, 300, device="cuda")
    L[0] = float("-inf")
    L[1] = float("nan")
    L[2] = float("-inf")
    L[2, 250] = -60000.0
    L[3] = torch.finfo(torch.float32).min               # lowest values: an even row
    L[4, 17] = float("inf")
    L[5, :] = float("nan")
    L[5, 299] = -1.0
    u = f32([0.5, 0.5, 0.5, 0.5, 0.5, 0.999])
    for args in ((), (f32([1.0] * 6), torch.full((6,), 40, device="cuda"), f32([0.9] * 6), f32([0.01] * 6))):
        got = lrc.sample(L, u, *args).cpu().tolist()
        assert got[0] == got[1] == -1 and got[2] == 250 and got[4] == 17 and got[5] == 299
        assert got[3] == (150 if not args else 18)      # of 300; of 36 = 0.9 * 40
    H16 = torch.full((1, 64), -65504.0, dtype=torch.float16, device="cuda")
    H16[0, 5] = 0.0
    assert lrc.sample(H16, f32([0.9])).item() == 5


def test_sample_filters_at_their_ends(lrc):
    L = torch.log(torch.tensor([[0.1, 0.4, 0.2, 0.3]] * 6, device="cuda"))
    u = f32([0.99] * 6)
    p = f32([0.0, -1.0, float("nan"), 2.0, 1e-9, 1.0])
    assert lrc.sample(L, u, top_p=p).cpu().tolist() == [1, 1, 3, 3, 1, 3]
    mp = f32([0.0, -1.0, float("nan"), 2.0, 0.6, 1.0])
    assert lrc.sample(L, u, min_p=mp).cpu().tolist() == [3, 3, 3, 1, 3, 1]
    k = torch.tensor([0, -5, 1, 2, 4, 2 ** 62], device="cuda")
    assert lrc.sample(L, u, top_k=k).cpu().tolist() == [3, 3, 1, 3, 3, 3]


def test_sample_pitch_alignment_and_stream(lrc):
    rng = np.random.default_rng(6)
    for prec in DT:
        big = rows_of(rng, 7, 3001, prec)
        u = torch.rand(7, device="cuda")
        for part in (big[:, 1:2990], big[:, :1000], big[2:5, 5:6]):
            n = part.shape[0]
            assert torch.equal(lrc.sample(part, u[:n].contiguous()), lrc.sample(part.contiguous(), u[:n].contiguous()))
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            out = lrc.sample(big, u)
        st.synchronize()
        assert torch.equal(out, lrc.sample(big, u))
    assert lrc.sample(torch.empty(0, 9, device="cuda"), torch.empty(0, device="cuda")).shape == (0,)


def test_sample_frequencies(lrc):
    """Evenly spaced u over one row: the counts are the probabilities to within one draw."""
    rng = np.random.default_rng(11)
    N, V = 2000, 700
    l = torch.from_numpy(rng.normal(size=V)).float().cuda()
    u = f32((np.arange(N) + 0.5) / N)
    got = lrc.sample(l.expand(N, V).contiguous(), u).cpu().numpy()
    q = np.exp(l.double().cpu().numpy())
    q /= q.sum()
    assert abs(np.bincount(got, minlength=V) - N * q).max() <= 1.01
    assert (np.diff(got) >= 0).all()
