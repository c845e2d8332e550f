"""The norm, the 8-bit product, the adapters and the verification as a step uses them: one after the other, captured and
replayed, on streams of their own, and with more rows than one workgroup sorts.

The chain's stages are each held to the 64-bit formula of what the stage before gave, with that stage's own tolerance
(those of its test file)."""
import numpy as np
import pytest

import test_gpu_adapter as TA
import test_gpu_q4_e4m3 as TQ
from oracle import head as H
from oracle import step as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def host(t):
    return t.double().cpu().numpy()


def chain(lrc, x, residual, weight, codes, scales, factors, A, B, ids, c, drafts, u):
    """(every stage's output) of one step's tail: norm in 8 bits, the compressed projection to the vocabulary, adapters
    beside it, the drafts' check"""
    R, D = drafts.shape
    y, t, h = lrc.rms_norm_e4m3(x, weight, residual=residual)
    z = lrc.q4_apply(codes, scales, y, 64, factors, out_dtype=x.dtype, x_scales=t)
    a = lrc.adapter_apply(h, A, B, ids, scale=c, base=z)
    tokens, accepted = lrc.verify(a.view(R, D + 1, -1), drafts, u, temperature=torch.zeros(R, device="cuda"))
    return y, t, h, z, a, tokens, accepted


def step(seed, R, D, n, V, k, prec):
    rng = np.random.default_rng(seed)
    rows = R * (D + 1)
    rand = lambda *s, size=1.0: torch.from_numpy(rng.normal(size=s) * size).to(DT[prec]).cuda()  # noqa: E731
    codes = rng.integers(0, 16, (V, n))
    scales = torch.from_numpy(rng.uniform(0.01, 0.05, (V, -(-n // 64)))).half()
    W = H.weights(codes, scales.double().numpy(), 64)
    factors = tuple(torch.from_numpy(rng.normal(size=s) * n ** -0.5).half().cuda() for s in ((V, k), (k,), (n, k)))
    q = TA.problem(seed, rows, V, n, 8, 5, "any", prec)
    return dict(x=rand(rows, n), residual=rand(rows, n), weight=rand(n), codes=torch.from_numpy(H.pack(codes)).cuda(),
                scales=scales.cuda(), factors=factors, A=q["A"], B=q["B"], ids=q["ids"], c=q["scale"],
                drafts=torch.zeros(R, D, dtype=torch.int64, device="cuda"), u=torch.rand(R, D + 1, device="cuda")), W, q


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("R,D,n,V,k", [(1, 0, 200, 515, 7), (3, 3, 640, 1003, 65), (12, 5, 515, 300, 12), (40, 4, 256, 700, 33)])
def test_a_step(lrc, prec, R, D, n, V, k):
    p, W, q = step(1, R, D, n, V, k, prec)
    # drafts that hold at some places and not at others
    a = chain(lrc, **p)[4]
    best = a.float().cpu().numpy().argmax(1).reshape(R, D + 1)
    drafts, want, count = best[:, :D].copy(), np.full((R, D + 1), -1), np.zeros(R, np.int64)
    for r in range(R):
        stop = r % (D + 1)
        if stop < D:
            drafts[r, stop] = (best[r, stop] + 1) % V
        want[r, :stop + 1], count[r] = best[r, :stop + 1], stop
    p["drafts"] = torch.from_numpy(drafts.astype(np.int64)).cuda()
    y, t, h, z, a, tokens, accepted = chain(lrc, **p)

    eps = torch.finfo(DT[prec]).eps / 2
    hd = (p["x"].float() + p["residual"].float()).to(DT[prec])
    assert torch.equal(h, hd)
    Y, _ = O.rms_norm(host(h), host(p["weight"]))
    td = np.abs(Y).max(1) / 448
    assert np.all(np.abs(host(t) - td) <= (n + 16) * U * td)
    # e4m3's half step, and the sum's error that may move a value over a rounding's edge: one step of it on top
    assert np.all(np.abs(host(y.float()) * td[:, None] - Y) <= (2.0 ** -4 + 2 * (n + 16) * U) * np.abs(Y) + td[:, None] * 2.0 ** -10 * (1 + 2 ** -6))
    TQ.check(z, W, y, t, p["factors"], prec)
    q = dict(q, X=h, base=z)
    (Ya, bY) = TA.bounds(q, prec)[0]
    TA.near(a, (Ya, bY), prec, "adapters")
    assert np.array_equal(tokens.cpu().numpy(), want) and np.array_equal(accepted.cpu().numpy(), count)
    assert eps < 1


def test_the_step_and_its_gradient_twice(lrc):
    """Every call repeats itself bit for bit."""
    p, _, q = step(2, 30, 5, 515, 1003, 33, "bf16")
    for one, two in zip(chain(lrc, **p), chain(lrc, **p)):
        assert torch.equal(one.view(torch.uint8), two.view(torch.uint8))
    for x, w in ((p["x"], p["weight"]), (p["x"].float(), p["weight"].float())):
        y, h, rstd = lrc.rms_norm(x, w, stats=True)
        for one, two in zip(*(lrc.rms_norm_backward(y, h, w, rstd, dsum=x) for _ in range(2))):
            assert torch.equal(one, two)


# ------------------------------------------------------------------- captured --

def replayed(lrc, call, fresh, grow, backs=lambda o: o):
    """call() -> outputs of the captured inputs; fresh() renews the inputs; grow() is a larger call on the same stream."""
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    same = lambda a, b: all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))  # noqa: E731
    with torch.cuda.stream(st):
        call()
        st.synchronize()
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            out = call()
        grow(1)                                             # two graphs, the second one's scratch larger or equal
        st.synchronize()
        with torch.cuda.graph(other, stream=st):
            out2 = call()
        for size in (1, 2, 4):
            fresh()
            graph.replay()
            st.synchronize()
            want = [t.clone() for t in call()]
            assert same(out, want)
            grow(size)
            st.synchronize()
            trash = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]
            fresh()
            other.replay()
            graph.replay()
            st.synchronize()
            got, got2 = [t.clone() for t in out], [t.clone() for t in out2]
            want = call()
            assert same(got, want) and same(got2, want)
            del trash


@pytest.mark.parametrize("rows,n", [(1, 2048), (40, 515), (1500, 640), (5, 40000)])
def test_norm_replayed(lrc, rows, n):
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, r, w, dy, big = rand(rows, n), rand(rows, n), rand(n), rand(rows, n), rand(4 * rows + 4000, n)
    torch.cuda.synchronize()

    def call():
        y, h, rstd = lrc.rms_norm(x, w, residual=r, stats=True)
        c, t, _ = lrc.rms_norm_e4m3(x, w, residual=r)
        return (y, h, rstd, c, t) + tuple(lrc.rms_norm_backward(dy, h, w, rstd, dsum=x))

    def grow(size):
        y, h, rstd = lrc.rms_norm(big[:rows + 1000 * size], w, stats=True)
        lrc.rms_norm_backward(y, h, w, rstd)

    def fresh():
        for t in (x, r, dy):
            t.normal_(generator=g)

    replayed(lrc, call, fresh, grow)


@pytest.mark.parametrize("rows,m,n,k", [(1, 515, 300, 8), (48, 300, 515, 17), (700, 130, 257, 40), (9000, 33, 40, 5)])
@pytest.mark.parametrize("prec", ["fp16", "fp32"])
def test_adapters_replayed(lrc, rows, m, n, k, prec):
    g = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[prec])  # noqa: E731
    count = 6
    X, A, B, base, dY, dbase = rand(rows, n), rand(count, k, n), rand(count, m, k), rand(rows, m), rand(rows, m), rand(rows, n)
    ids = torch.zeros(rows, dtype=torch.int64, device="cuda")
    big = rand(4 * rows + 800, n)
    bids = torch.randint(-1, count + 1, (len(big),), generator=g, device="cuda")
    torch.cuda.synchronize()

    def call():
        Y, H = lrc.adapter_apply(X, A, B, ids, base=base, hidden=True)
        return (Y, H) + tuple(lrc.adapter_backward(dY, X, A, B, ids, H, base=dbase))

    def grow(size):
        b = rows * size + 200 * size
        Y, H = lrc.adapter_apply(big[:b], A, B, bids[:b], hidden=True)
        lrc.adapter_backward(Y, big[:b], A, B, bids[:b], H)

    def fresh():
        for t in (X, base, dY, dbase):
            t.normal_(generator=g)
        ids.random_(-1, count + 1, generator=g)

    replayed(lrc, call, fresh, grow)


@pytest.mark.parametrize("R,D,V", [(1, 4, 65536), (6, 3, 5003)])
def test_verification_replayed(lrc, R, D, V):
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda") * 2  # noqa: E731
    L, Q, u = rand(R, D + 1, V), rand(R, D, V), torch.rand(R, D + 1, generator=g, device="cuda")
    d = torch.zeros(R, D, dtype=torch.int64, device="cuda")
    p, big = torch.full((R,), 0.9, device="cuda"), rand(16, 9, V)
    bd, bu = torch.zeros(16, 8, dtype=torch.int64, device="cuda"), torch.rand(16, 9, generator=g, device="cuda")
    torch.cuda.synchronize()

    def fresh():
        L.normal_(generator=g).mul_(2)
        Q.copy_(L[:, :D]).add_(torch.randn(R, D, V, generator=g, device="cuda"), alpha=0.1)
        u.uniform_(generator=g)
        d.copy_(Q.argmax(2))

    replayed(lrc, lambda: lrc.verify(L, d, u, draft_logits=Q, top_p=p), fresh, lambda size: lrc.verify(big[:4 * size], bd[:4 * size], bu[:4 * size]))


@pytest.mark.parametrize("b,m,n,k", [(1, 512, 1024, 9), (20, 700, 640, 33), (200, 512, 515, 65)])
def test_8_bit_product_replayed(lrc, b, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    codes, scales = lrc.q4_quantize(rand(m, n), group=128)
    F = (rand(m, k).half(), rand(k).half(), rand(n, k).half())
    X, t, big = (rand(b, n) * 50).to(torch.float8_e4m3fn), torch.rand(b, generator=g, device="cuda"), rand(4 * 700, n).to(torch.float8_e4m3fn)
    bt = torch.rand(4 * 700, generator=g, device="cuda")
    torch.cuda.synchronize()

    def fresh():
        X.copy_(rand(b, n) * 50)
        t.uniform_(generator=g)

    replayed(lrc, lambda: (lrc.q4_apply(codes, scales, X, 128, F, x_scales=t),), fresh,
             lambda size: lrc.q4_apply(codes, scales, big[:size * 700], 128, F, x_scales=bt[:size * 700]))


def test_two_streams_at_once(lrc):
    """Calls of two streams have a workspace each."""
    p, _, _ = step(5, 20, 5, 640, 1003, 33, "bf16")
    p2, _, _ = step(6, 30, 3, 515, 700, 17, "bf16")
    want, want2 = chain(lrc, **p), chain(lrc, **p2)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        with torch.cuda.stream(a):
            got.append((chain(lrc, **p), want))
        with torch.cuda.stream(b):
            got.append((chain(lrc, **p2), want2))
    torch.cuda.synchronize()
    for one, two in got:
        for x, y in zip(one, two):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


# ------------------------------------------------------------------ many rows --

@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,count,kind", [(8192, 40, "any"), (8193, 40, "any"), (20011, 300, "any"), (20011, 1, "one"), (9000, 3, "none"),
                                             (12345, 70000, "any")])
def test_adapters_of_many_rows(lrc, prec, rows, count, kind):
    q = TA.problem(9, rows, 37, 41, 3, count, kind, prec)
    if count <= 300:
        Y, Hd, dX, dA, dB = TA.bounds(q, prec)
    got, hidden = lrc.adapter_apply(q["X"], q["A"], q["B"], q["ids"], scale=q["scale"], base=q["base"], hidden=True)
    grads = lrc.adapter_backward(q["dY"], q["X"], q["A"], q["B"], q["ids"], hidden, scale=q["scale"], base=q["dbase"])
    if count <= 300:
        TA.near(hidden, Hd, "fp32", "hidden")
        TA.near(got, Y, prec, "Y")
        for x, w, what in zip(grads, (dX, dA, dB), ("dX", "dA", "dB")):
            TA.near(x, w, prec, what)
    # a row depends on the rows beside it in nothing but its sums' order: 41 products of size 41^-1/2 and a rounding each
    some = torch.from_numpy(np.random.default_rng(3).choice(rows, 2000, replace=False)).cuda()
    Ys, Hs = lrc.adapter_apply(q["X"][some], q["A"], q["B"], q["ids"][some], scale=q["scale"], base=q["base"][some], hidden=True)
    eps = torch.finfo(DT[prec]).eps
    assert torch.allclose(Hs, hidden[some], rtol=0, atol=1e-5)
    assert torch.allclose(Ys.float(), got[some].float(), rtol=2 * eps, atol=1e-4)


def test_offsets_past_32_bits(lrc):
    """Rows whose elements lie past 2^31 (norm, adapters, verification): pitched rows of one large array."""
    n, ld = 1024, 1 << 22
    rows = 1030                                             # last row begins at 4.3e9 elements
    big = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = big.view(rows, ld)[:, :n]
    g = torch.Generator(device="cuda").manual_seed(7)
    small = torch.randn(rows, n, generator=g, device="cuda").bfloat16()
    x.copy_(small)
    w = torch.randn(n, generator=g, device="cuda").bfloat16()
    for one, two in zip(lrc.rms_norm_e4m3(x, w)[:2], lrc.rms_norm_e4m3(small, w)[:2]):
        assert torch.equal(one.view(torch.uint8), two.view(torch.uint8))
    y, h, rstd = lrc.rms_norm(small, w, stats=True)
    for one, two in zip(lrc.rms_norm_backward(x, x, w, rstd, dsum=x), lrc.rms_norm_backward(small, small, w, rstd, dsum=small)):
        assert torch.equal(one, two)
    A, B = torch.randn(3, 8, n, generator=g, device="cuda").bfloat16(), torch.randn(3, n, 8, generator=g, device="cuda").bfloat16()
    ids = torch.randint(-1, 3, (rows,), generator=g, device="cuda")
    Y, Hd = lrc.adapter_apply(small, A, B, ids, base=small, hidden=True)
    Yb, Hb = lrc.adapter_apply(x, A, B, ids, base=x, hidden=True)
    assert torch.equal(Y, Yb) and torch.equal(Hd, Hb)
    for one, two in zip(lrc.adapter_backward(x, x, A, B, ids, Hd, base=x), lrc.adapter_backward(small, small, A, B, ids, Hd, base=small)):
        assert torch.equal(one, two)
    for r in (rows - 4, rows - 64):                         # few rows, far away
        assert torch.equal(lrc.adapter_apply(x[r:], A, B, ids[r:]), lrc.adapter_apply(small[r:], A, B, ids[r:]))
    R, D = 206, 4
    d, u = small.view(R, D + 1, n)[:, :D].argmax(2), torch.rand(R, D + 1, generator=g, device="cuda")
    L = x.unflatten(0, (R, D + 1))
    one, two = lrc.verify(L, d, u, draft_logits=L[:, :D]), lrc.verify(small.view(R, D + 1, n), d, u, draft_logits=small.view(R, D + 1, n)[:, :D])
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


# ---------------------------------------------------------------- many of them --

@pytest.mark.parametrize("R,D,V", [(70000, 1, 5), (1, 3000, 3), (2, 65536, 2), (5000, 7, 2)])
def test_many_requests_and_drafts(lrc, R, D, V):
    """Greedy: drafts hold up to the first that is not its row's largest logit."""
    g = torch.Generator(device="cuda").manual_seed(R)
    L = torch.randn(R, D + 1, V, generator=g, device="cuda")
    best = L.argmax(2)
    stop = torch.randint(0, D + 1, (R,), generator=g, device="cuda")
    drafts = best[:, :D].clone()
    at = torch.arange(D, device="cuda")[None] == stop[:, None]
    drafts[at] = (drafts[at] + 1) % V
    tokens, accepted = lrc.verify(L, drafts, torch.rand(R, D + 1, generator=g, device="cuda"), temperature=torch.zeros(R, device="cuda"))
    behind = torch.arange(D + 1, device="cuda")[None] > stop[:, None]
    assert torch.equal(accepted, stop) and torch.equal(tokens, best.masked_fill(behind, -1))


@pytest.mark.parametrize("rows,n", [(300000, 4), (70000, 1), (2100000, 3), (3, 300001)])
def test_norm_of_many_rows_and_of_long_ones(lrc, rows, n):
    """Against 64 bits: n + 8 roundings of the sum (halved by the root), four of the product."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = torch.randn(rows, n, generator=g, device="cuda"), torch.randn(rows, n, generator=g, device="cuda")
    w = torch.randn(n, generator=g, device="cuda")
    y, h, rstd = lrc.rms_norm(x, w, stats=True, eps=1e-3)
    X, W, DY = x.double(), w.double(), dy.double()
    r = (X * X).mean(1, keepdim=True).add(1e-3).rsqrt()
    bound = (n + 16) * U
    assert ((y.double() - X * r * W).abs() <= bound * (X * r * W).abs() + 1e-38).all()
    dx, dw = lrc.rms_norm_backward(dy, h, w, rstd)
    s = (DY * W * X * r).mean(1, keepdim=True)
    size = (DY * W * X * r).abs().mean(1, keepdim=True)
    want, scale = r * (DY * W - X * r * s), r * ((DY * W).abs() + (X * r).abs() * size)
    assert ((dx.double() - want).abs() <= 2 * bound * scale + 1e-38).all()
    want, scale = (DY * X * r).sum(0), (DY * X * r).abs().sum(0)
    assert ((dw.double() - want).abs() <= (bound + (rows + 16) * U) * scale).all()


def test_adapters_of_a_great_many_rows(lrc):
    """More rows than two bytes name; whole values, so that every sum is exact."""
    rows, n, m, k, count = 300000, 4, 5, 2, 7
    g = torch.Generator(device="cuda").manual_seed(11)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda").float()  # noqa: E731
    X, A, B, base, dY = whole(rows, n), whole(count, k, n), whole(count, m, k), whole(rows, m), whole(rows, m)
    ids = torch.randint(-1, count + 1, (rows,), generator=g, device="cuda")
    Y, Hd = lrc.adapter_apply(X, A, B, ids, base=base, hidden=True)
    dX, dA, dB = lrc.adapter_backward(dY, X, A, B, ids, Hd)
    wH, wY, wX = torch.zeros(rows, k, device="cuda"), base.clone(), torch.zeros(rows, n, device="cuda")
    for a in range(count):
        i = ids == a
        wH[i] = X[i] @ A[a].T
        wY[i] += wH[i] @ B[a].T
        dh = dY[i] @ B[a]
        wX[i] = dh @ A[a]
        assert torch.equal(dA[a], dh.T @ X[i]) and torch.equal(dB[a], dY[i].T @ wH[i])
    assert torch.equal(Hd, wH) and torch.equal(Y, wY) and torch.equal(dX, wX)


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
def test_gradients_without_rows(lrc, prec):
    """Empty tensors, without memory of their own, and weights whose gradients are 0."""
    new = lambda *s: torch.empty(*s, dtype=DT[prec], device="cuda")  # noqa: E731
    A, B, w = new(3, 5, 20).fill_(1), new(3, 30, 5).fill_(1), new(20).fill_(1)
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    dX, dA, dB = lrc.adapter_backward(new(0, 30), new(0, 20), A, B, ids, torch.empty(0, 5, device="cuda"))
    assert dX.shape == (0, 20) and not dA.any() and not dB.any()
    assert lrc.adapter_apply(new(0, 20), A, B, ids).shape == (0, 30)
    dx, dw = lrc.rms_norm_backward(new(0, 20), new(0, 20), w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 20) and not dw.any()


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,n", [(3000, 515), (2047, 5003), (700, 9000), (300, 17000), (40, 8)])
def test_norm_gradient_in_place(lrc, prec, rows, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[prec])  # noqa: E731
    dy, h, ds, w = rand(rows, n), rand(rows, n), rand(rows, n), rand(n)
    rstd = lrc.rms_norm(h, w, stats=True)[2]
    want, dw = lrc.rms_norm_backward(dy, h, w, rstd, dsum=ds)
    for mine in (0, 1):
        a, b = dy.clone(), ds.clone()
        got, dw2 = lrc.rms_norm_backward(a, h, w, rstd, dsum=b, dx=(a, b)[mine])
        assert torch.equal(got, want) and torch.equal(dw, dw2)
