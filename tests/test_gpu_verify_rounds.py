"""Verification whose rows are passed in several rounds (as many places at first as fill the compute units, then twice as many
each time), with draft logits, against exact integers: requests that end in every round, and requests whose drafts end before
a round's first place."""
import numpy as np
import pytest

from test_gpu_verify import f32, i64, request

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("R,D,V,first", [(48, 5, 257, 2), (70, 6, 40, 1), (140, 8, 33, 1), (130, 3, 1009, 1), (20, 13, 50, 6)])
@pytest.mark.parametrize("sure", [False, True])
def test_rounds_against_integers(lrc, prec, R, D, V, first, sure):
    rng = np.random.default_rng([R, D, V, sure])
    made = [request(rng, D, V, prec, r % 7 == 3, 0.0, sure) for r in range(R)]
    taken, have = [x[6] for x in made], [next((j for j, d in enumerate(x[3]) if not 0 <= d < V), D) for x in made]
    # a round's places: from `at` on, `some` of them
    at, some, rounds = 0, first, 0
    while at <= D:
        assert any(at <= n < at + some for n in taken) and (at == 0 or any(h < at for h in have)), (at, some)
        at, some, rounds = at + some, 2 * some, rounds + 1
    assert rounds > 1
    P = torch.stack([x[0] for x in made]).cuda()
    Q = None if sure else torch.stack([x[1] for x in made]).cuda()
    T, k, p, mp = zip(*[x[2] for x in made])
    drafts, u = i64([x[3] for x in made]), f32([x[4] for x in made])
    args = dict(temperature=f32(T), top_k=i64(k), top_p=f32(p), min_p=f32(mp))
    tokens, accepted = lrc.verify(P, drafts, u, draft_logits=Q, **args)
    assert accepted.cpu().tolist() == taken
    assert tokens.cpu().tolist() == [x[5] for x in made]
    # each request by itself, in a round of its own
    for r in (0, 3, R - 1):
        one = lrc.verify(P[r:r + 1], drafts[r:r + 1], u[r:r + 1], draft_logits=None if sure else Q[r:r + 1],
                         **{n: v[r:r + 1] for n, v in args.items()})
        assert torch.equal(one[0], tokens[r:r + 1]) and torch.equal(one[1], accepted[r:r + 1])
