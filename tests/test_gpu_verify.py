"""Verification of drafted tokens against exact integers (oracle/step.py), the weights from the oracle's filters.

Tokens are whole numbers, so the tests decide where rounding cannot: thresholds of the filters lie between two tokens,
numbers that accept a draft lie 1e-3 away from p / q, and the drawn token's number in the middle of an interval of
1e-4 or more (weights are binary32 values with relative errors below 1e-5)."""
import numpy as np
import pytest

from oracle import head as H
from oracle import step as O

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


def i64(x):
    return torch.tensor(np.asarray(x, np.int64), device="cuda")


def weights(l, T, k, p, mp):
    """Whole weights of a row of logits under the request's parameters."""
    l = np.where(np.isnan(l), -np.inf, l)
    if l.max() == -np.inf:
        return np.zeros(len(l))
    if not T > 0:
        w = np.zeros(len(l))
        w[l.argmax()] = 2.0 ** 31
        return w
    return H.sample_kept(l, T, k, p, mp)[1]


def fits(rows, T, k, p, mp):
    """Whether the filters' thresholds are far from every token of the rows."""
    for l in rows:
        order, kept = H.sample_kept(l, T, k)
        ws = kept[order]
        ws = ws[ws > 0] / ws.sum()
        if p < 1 and np.abs(np.cumsum(ws) - p).min() < 2e-5:
            return False
        if mp > 0:
            w = np.exp((l - l.max()) / T)
            if np.abs(w / mp - 1).min() < 1e-4:
                return False
    return True


def request(rng, D, V, prec, greedy, masked, sure):
    """(target logits, draft logits, parameters, drafts, u, tokens, accepted) of one request."""
    while True:
        p = rng.normal(size=(D + 1, V)) * 2
        for r in range(D + 1):
            p[r, rng.integers(0, V, min(6, V))] += 5.0
        q = p[:D] + rng.normal(size=(D, V)) * 0.5
        if masked:
            gone = rng.random(V) < masked
            gone[rng.integers(0, V)] = False
            p[:, gone] = q[:, gone] = -np.inf
        P, Q = (torch.from_numpy(x).to(DT[prec]) for x in (p, q))
        hp, hq = P.double().numpy(), Q.double().numpy()
        T = 0.0 if greedy else float(np.float32(rng.uniform(0.6, 1.4)))
        k = int(rng.choice([0, 1, 3, 20, 300, V]))
        tp = float(np.float32(rng.uniform(0.3, 0.95))) if rng.random() < 0.5 else 1.0
        mp = float(np.float32(rng.uniform(0.002, 0.2))) if rng.random() < 0.4 else 0.0
        if greedy or fits(list(hp) + list(hq), T, k, tp, mp):
            break
    wp = np.stack([weights(l, T, k, tp, mp) for l in hp])
    wq = np.stack([weights(l, T, k, tp, mp) for l in hq]) if D else np.zeros((0, V))
    have = int(rng.integers(0, D + 1)) if rng.random() < 0.3 else D
    drafts, u = np.full(D, -1), np.zeros(D + 1, np.float32)
    if have < D and rng.random() < 0.5:
        drafts[have] = V                                   # past the vocabulary: no token either
        drafts[have + 1:] = 0                              # what follows does not count
    for j in range(have):
        drafts[j] = rng.choice(V, p=wq[j] / wq[j].sum()) if rng.random() < 0.8 else rng.integers(0, V)
        q = wq[j] if not sure else (np.arange(V) == drafts[j])
        ratio = 0.0 if wp[j][drafts[j]] == 0 else np.inf if q[drafts[j]] == 0 else \
            wp[j][drafts[j]] / wp[j].sum() / (q[drafts[j]] / q.sum())
        accept = rng.random() < 0.75
        u[j] = min(rng.uniform(0, 1) if ratio in (0.0, np.inf) else ratio * (1 - 1e-3) * rng.uniform(0, 1) if accept
                   else ratio * (1 + 1e-3), 1 - 2.0 ** -24)
        if 0.999 <= ratio <= 1.001:
            u[j] = 0.5
    # the drawn token: the middle of a wide interval
    u[D] = 0.5
    _, taken = O.verify(wp, drafts, u, None if sure else wq)
    if taken < D and 0 <= drafts[taken] < V:
        q = (np.arange(V) == drafts[taken]) * 1.0 if sure else wq[taken] / wq[taken].sum()
        rest = np.maximum(wp[taken] / wp[taken].sum() - q, 0)
        if rest.sum() < 1e-3:
            return request(rng, D, V, prec, greedy, masked, sure)      # little is left, mostly roundings: another one
    else:
        rest = wp[taken]
    c = rest / rest.sum()
    wide = np.flatnonzero(c >= 2e-4)
    if len(wide) == 0:
        return request(rng, D, V, prec, greedy, masked, sure)
    j = int(rng.choice(wide))
    u[D] = c[:j].sum() + c[j] / 2
    tokens, n = O.verify(wp, drafts, u, None if sure else wq)
    assert tokens[n] == j
    return P, Q, (T, k, tp, mp), drafts, u, tokens, n


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("R,D,V", [(1, 1, 1), (3, 0, 50), (4, 2, 5), (30, 3, 257), (6, 8, 1003), (3, 5, 8192), (2, 2, 32003),
                                   (1, 70, 40)])
@pytest.mark.parametrize("masked,sure", [(0.0, False), (0.0, True), (0.7, False)])
def test_against_integers(lrc, prec, R, D, V, masked, sure):
    rng = np.random.default_rng([R, D, V])
    made = [request(rng, D, V, prec, r % 5 == 4, masked, sure) for r in range(R)]
    P = torch.stack([x[0] for x in made]).cuda()
    Q = torch.stack([x[1] for x in made]).cuda() if D else None
    T, k, p, mp = zip(*[x[2] for x in made])
    tokens, accepted = lrc.verify(P, i64([x[3] for x in made]).view(R, D), f32([x[4] for x in made]),
                                  draft_logits=None if sure else Q, temperature=f32(T), top_k=i64(k), top_p=f32(p), min_p=f32(mp))
    assert accepted.cpu().tolist() == [x[6] for x in made]
    assert tokens.cpu().tolist() == [x[5] for x in made]


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
def test_without_drafts_it_is_the_draw(lrc, prec):
    g = torch.Generator(device="cuda").manual_seed(3)
    R, V = 50, 20011
    L = (torch.randn(R, V, generator=g, device="cuda") * 3).to(DT[prec])
    L[7] = float("-inf")
    L[8, 100:200] = float("inf")
    L[9, :5000] = 2.0
    L[10] = float("nan")
    u = torch.rand(R, generator=g, device="cuda")
    T = torch.rand(R, generator=g, device="cuda") + 0.5
    T[::6] = 0.0
    k = torch.randint(-1, 400, (R,), generator=g, device="cuda")
    k[9], T[9] = 1234, 1.0
    p = torch.rand(R, generator=g, device="cuda") + 0.3
    mp = torch.rand(R, generator=g, device="cuda") * 0.2 - 0.1
    want = lrc.sample(L, u, T, k, p, mp)
    none = torch.empty(R, 0, dtype=torch.int64, device="cuda")
    tokens, accepted = lrc.verify(L[:, None], none, u[:, None].contiguous(), temperature=T, top_k=k, top_p=p, min_p=mp)
    assert torch.equal(tokens[:, 0], want) and not accepted.any()
    # and behind drafts that are certain and accepted: u = 0 takes any draft that the target keeps
    first = lrc.sample(L, u * 0.9, T, k, p, mp)
    ok = first >= 0
    both = torch.stack([L, L], 1)
    w = torch.stack([torch.zeros_like(u), u], 1).contiguous()
    tokens, accepted = lrc.verify(both, first[:, None].contiguous(), w, temperature=T, top_k=k, top_p=p, min_p=mp)
    assert torch.equal(accepted, ok.long())
    assert torch.equal(tokens[ok], torch.stack([first, want], 1)[ok])
    assert (tokens[~ok] == -1).all()


def test_numbers_at_and_past_the_ends(lrc):
    """u outside [0, 1) moves to the nearer end: the smallest takes every draft that the target keeps, the largest
    none that the draft model names more often than the target."""
    L = torch.tensor([0.0, 1.0, 2.0, float("-inf")], device="cuda").repeat(6, 2, 1)
    Q = torch.tensor([3.0, 1.0, 0.0, 0.0], device="cuda").repeat(6, 1, 1)
    d = i64([[0]] * 6)
    u = f32([[0.0, 0.5], [-3.0, 0.5], [float("nan"), 0.5], [1.0, 0.999999], [7.0, 5.0], [0.999999, -1.0]])
    tokens, accepted = lrc.verify(L, d, u, draft_logits=Q)
    assert accepted.cpu().tolist() == [1, 1, 1, 0, 0, 0]
    # what the target has above the draft: tokens 1 and 2
    assert tokens.cpu().tolist() == [[0, 2], [0, 2], [0, 2], [2, -1], [2, -1], [1, -1]]
    # a draft that neither the target nor the draft model keeps is not taken, one that only the target keeps is
    tokens, accepted = lrc.verify(L[:2], i64([[3], [2]]), f32([[0.0, 0.0], [0.99, 0.0]]),
                                  draft_logits=torch.tensor([0.0, 0.0, float("-inf"), float("-inf")], device="cuda").repeat(2, 1, 1))
    assert accepted.cpu().tolist() == [0, 1] and tokens.cpu().tolist() == [[2, -1], [2, 0]]


def test_rows_that_weigh_nothing(lrc):
    ninf, inf, nan = float("-inf"), float("inf"), float("nan")
    L = torch.tensor([[[ninf] * 3, [0.0] * 3], [[0.0, 1, 2], [nan] * 3], [[inf, 0, inf], [0, inf, 0]], [[0.0, 0, 0]] * 2],
                     device="cuda")
    Q = torch.tensor([[[0.0] * 3], [[0.0] * 3], [[inf, 0, inf]], [[ninf, nan, ninf]]], device="cuda")
    tokens, accepted = lrc.verify(L, i64([[0], [2], [2], [1]]), f32([[0.0, 0.0], [0.0, 0.0], [0.5, 0.0], [0.9, 0.5]]), draft_logits=Q)
    # nothing to accept against; nothing behind the draft; equal infinities; a draft row of nothing rejects
    assert accepted.cpu().tolist() == [0, 1, 1, 0]
    assert tokens.cpu().tolist() == [[-1, -1], [2, -1], [2, 1], [1, -1]]


def test_equal_distributions_with_ties(lrc):
    """Equal rows accept every kept draft; a tie outside the top-k prefix is not kept."""
    V = 3000
    L = torch.full((3, 2, V), 1.0, device="cuda")
    k = i64([5, 5, 5])
    d = i64([[4], [5], [0]])
    u = f32([[0.999, 0.999], [0.0, 0.1], [0.999, 0.0]])
    tokens, accepted = lrc.verify(L, d, u, draft_logits=L[:, :1].contiguous(), top_k=k)
    assert accepted.cpu().tolist() == [1, 0, 1]
    assert tokens.cpu().tolist() == [[4, 4], [0, -1], [0, 0]]      # the rejected one: nothing is left, the target's draw
    for dt in (torch.float16, torch.bfloat16):
        t2, a2 = lrc.verify(L.to(dt), d, u, draft_logits=L[:, :1].to(dt).contiguous(), top_k=k)
        assert torch.equal(t2, tokens) and torch.equal(a2, accepted)
    # ties that no list holds: 30000 equal logits
    L = torch.full((2, 2, 30000), 1.0, device="cuda")
    tokens, accepted = lrc.verify(L, i64([[19999], [20000]]), f32([[0.5, 0.99999], [0.0, 0.0]]),
                                  draft_logits=L[:, :1].contiguous(), top_k=i64([20000, 20000]))
    assert accepted.cpu().tolist() == [1, 0] and tokens.cpu().tolist() == [[19999, 19999], [0, -1]]


def test_pitches_and_repeatability(lrc):
    g = torch.Generator(device="cuda").manual_seed(4)
    R, D, V = 20, 3, 5001
    big = torch.randn(R + 1, D + 2, V + 9, generator=g, device="cuda") * 3
    L = big[1:, :D + 1, 3:3 + V]
    Q = big[:R, 1:, 5:5 + V][:, :D]
    d = torch.randint(0, V, (R, D), generator=g, device="cuda")
    d[:, 0] = Q[:, 0].argmax(1)
    u = torch.rand(R, D + 1, generator=g, device="cuda")
    p = torch.full((R,), 0.9, device="cuda")
    a = lrc.verify(L, d, u, draft_logits=Q, top_p=p)
    b = lrc.verify(L.contiguous(), d, u, draft_logits=Q.contiguous(), top_p=p)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    one = lrc.verify(L[3:4], d[3:4], u[3:4], draft_logits=Q[3:4], top_p=p[3:4])
    assert torch.equal(one[0], a[0][3:4])
    empty = lrc.verify(L[:0], d[:0], u[:0], draft_logits=Q[:0])
    assert empty[0].shape == (0, D + 1) and empty[1].shape == (0,)


def test_tokens_follow_the_target(lrc):
    """The law of the first token, over many numbers, is the target's whatever the draft model: within five standard
    deviations of every frequency."""
    g = torch.Generator(device="cuda").manual_seed(5)
    V, N = 12, 200000
    p, q = torch.randn(V, generator=g, device="cuda"), torch.randn(V, generator=g, device="cuda")
    d = lrc.sample(q.repeat(N, 1), torch.rand(N, generator=g, device="cuda"))
    tokens, accepted = lrc.verify(p.expand(N, 2, V), d[:, None].contiguous(), torch.rand(N, 2, generator=g, device="cuda"),
                                  draft_logits=q.expand(N, 1, V))
    want = torch.softmax(p.double(), 0)
    got = torch.bincount(tokens[:, 0], minlength=V).double() / N
    assert ((got - want).abs() <= 5 * (want * (1 - want) / N).sqrt()).all()
    # and so is that of the token behind an accepted draft
    after = tokens[accepted == 1, 1]
    got = torch.bincount(after, minlength=V).double() / len(after)
    assert ((got - want).abs() <= 5 * (want * (1 - want) / len(after)).sqrt()).all()
