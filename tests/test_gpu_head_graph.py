"""Captured output-head calls whose stream later takes larger calls: the replays keep their scratch.  Every replay is
compared with the eager result, with eager work and synchronizations between the replays."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def replayed(lrc, call, fresh, grow, warm):
    """call() -> output of the captured inputs; fresh() renews them; grow() is a larger call."""
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        if warm:
            call()
            st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out = call()
        for size in (1, 2, 4):
            fresh()
            graph.replay()
            st.synchronize()
            assert torch.equal(out, call())
            grow(size)
            st.synchronize()
            trash = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
            fresh()
            graph.replay()
            st.synchronize()
            got = out.clone()
            assert torch.equal(got, call())
            del trash


@pytest.mark.parametrize("warm", [True, False])
@pytest.mark.parametrize("b", [1, 20])
def test_product_replayed_after_larger_calls(lrc, warm, b):
    g = torch.Generator(device="cuda").manual_seed(b)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    m, n, k = 2048, 1024, 33
    codes, scales = lrc.q4_quantize(rand(m, n), group=64)
    F = (rand(m, k).half(), rand(k).half(), rand(n, k).half())
    X, big = rand(b, n).bfloat16(), rand(4 * 700, n)
    torch.cuda.synchronize()
    replayed(lrc, lambda: lrc.q4_apply(codes, scales, X, 64, F), lambda: X.normal_(generator=g),
             lambda size: lrc.q4_apply(codes, scales, big[:size * 700], 64, F), warm)


@pytest.mark.parametrize("warm", [True, False])
def test_sampling_replayed_after_larger_calls(lrc, warm):
    g = torch.Generator(device="cuda").manual_seed(5)
    L = torch.randn(2, 128003, generator=g, device="cuda") * 3
    u = torch.rand(2, generator=g, device="cuda")
    k, p = torch.tensor([40, 0], device="cuda"), torch.tensor([0.9, 0.7], device="cuda")
    more = torch.randn(16, 131072, generator=g, device="cuda")
    w = torch.rand(16, device="cuda")
    torch.cuda.synchronize()

    def fresh():
        L.normal_(generator=g).mul_(3)
        u.uniform_(generator=g)

    replayed(lrc, lambda: lrc.sample(L, u, top_k=k, top_p=p), fresh, lambda size: lrc.sample(more[:4 * size], w[:4 * size]), warm)


def test_factor_apply_replayed_after_larger_calls(lrc):
    g = torch.Generator(device="cuda").manual_seed(6)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    U, s, V, X, big = rand(1000, 40), rand(40), rand(900, 40), rand(900, 64), rand(900, 4 * 1000)
    torch.cuda.synchronize()
    replayed(lrc, lambda: lrc.matrix_apply(U, s, V, X), lambda: X.normal_(generator=g),
             lambda size: lrc.matrix_apply(U, s, V, big[:, :size * 1000].contiguous()), True)
