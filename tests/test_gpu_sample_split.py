"""Sampling of few long rows (a row on several workgroups) against many (a workgroup a row): weights are whole numbers, so
the tokens are equal whatever the split.  Batches above 16 rows, and rows below 98304 logits, take the second way."""
import numpy as np
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


def rows_of_every_kind(g, V, prec):
    """Rows whose logits lie in every way that the kernels tell apart."""
    L = torch.randn(14, V, generator=g, device="cuda") * 2
    L[0] = float("-inf")
    L[1] = float("nan")
    L[2] = float("-inf")
    L[2, V - 1] = -60000.0
    L[3] = torch.finfo(DT[prec]).min
    L[4, V // 2] = float("inf")
    L[5, ::2] = float("nan")
    L[6] = 1.5                                       # every logit equal: no list holds them
    L[7, : V // 3] = float("-inf")
    L[8] = L[8].round()                              # thousands of ties a value
    L[9] *= 100.0
    L[10] *= 1e-3
    L[11, 0] = 40.0                                  # one token takes all
    L[12, :: 4097] = 9.0                             # the likeliest in every part
    L[13] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.999, float("-inf"), L[13])
    return L.to(DT[prec])


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("V", [20011, 98304, 131071, 200003])
def test_few_rows_draw_what_many_draw(lrc, prec, V):
    g = torch.Generator(device="cuda").manual_seed(V)
    L = rows_of_every_kind(g, V, prec)
    n = L.shape[0]
    many = L.repeat(10, 1)                           # a workgroup a row
    rng = np.random.default_rng(V)
    for trial in range(6):
        f = lambda x: torch.tensor(np.asarray(x, np.float32), device="cuda")  # noqa: E731
        u = f(rng.random(n))
        T = f(rng.choice([0.0, 0.3, 1.0, 1.7, 50.0], n))
        k = torch.tensor(rng.choice([0, 1, 7, 300, 5000, V], n), device="cuda")
        p = f(rng.choice([0.1, 0.5, 0.99, 1.0], n))
        mp = f(rng.choice([0.0, 0.02, 1.0], n))
        if trial == 0:
            T, k, p, mp = None, None, None, None
        rep = lambda x: None if x is None else x.repeat(10)  # noqa: E731
        want = lrc.sample(many, rep(u), rep(T), rep(k), rep(p), rep(mp))[:n]
        assert torch.equal(lrc.sample(L, u, T, k, p, mp), want)
        one = lambda x, r: None if x is None else x[r:r + 1]  # noqa: E731
        for r in range(0, n, 3):
            assert torch.equal(lrc.sample(L[r:r + 1], u[r:r + 1], one(T, r), one(k, r), one(p, r), one(mp, r)), want[r:r + 1])


def test_few_rows_in_a_replayed_graph(lrc):
    g = torch.Generator(device="cuda").manual_seed(1)
    L = torch.randn(3, 128003, generator=g, device="cuda") * 3
    u = torch.rand(3, generator=g, device="cuda")
    k = torch.tensor([0, 40, 0], device="cuda")
    p = torch.tensor([1.0, 0.9, 0.7], device="cuda")
    out = torch.empty(3, dtype=torch.int64, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        lrc.sample(L, u, top_k=k, top_p=p, out=out)    # the workspace is there before the capture
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            lrc.sample(L, u, top_k=k, top_p=p, out=out)
    for _ in range(4):
        L.normal_(generator=g).mul_(3)
        u.uniform_(generator=g)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, lrc.sample(L, u, top_k=k, top_p=p))
