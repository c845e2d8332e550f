"""Outputs and inputs of the step calls that the C interface lets a caller leave out (NULL), which the binding always gives:
what remains is bit for bit what the whole call gives."""
import itertools

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
CODE = {"fp32": 1, "fp16": 2, "bf16": 3}


@pytest.fixture(scope="module")
def lrc():
    from paper_2607_12969_amd import lrc as mod
    assert torch.cuda.is_available()
    mod.lib()
    return mod


def p(t):
    return None if t is None else t.data_ptr()


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,m,n,k,count", [(90, 70, 130, 12, 3), (1200, 130, 90, 40, 2), (300, 64, 72, 5, 40), (9000, 24, 40, 8, 5)])
@pytest.mark.parametrize("scaled,based", [(True, True), (False, False)])
def test_adapter_gradients_one_by_one(lrc, prec, rows, m, n, k, count, scaled, based):
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    R = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[prec])  # noqa: E731
    X, dY, A, B = R(rows, n), R(rows, m), R(count, k, n) * n ** -0.5, R(count, m, k) * k ** -0.5
    ids = torch.randint(-1, count + 1, (rows,), generator=g, device="cuda")
    scale = torch.rand(count, generator=g, device="cuda") + 0.5 if scaled else None
    base = R(rows, n) if based else None
    hidden = lrc.adapter_apply(X, A, B, ids, scale=scale, hidden=True)[1]
    whole = lrc.adapter_backward(dY, X, A, B, ids, hidden, scale=scale, base=base)
    for give in itertools.product((False, True), repeat=3):
        dX, dA, dB = (torch.full_like(t, 7.0) if on else None for on, t in zip(give, whole))
        lrc._launch(X.device, "lrc_adapter_backward", p(dY), m, p(X) if give[1] else None, n, p(A) if give[0] else None, p(B), p(ids), p(scale),
                    p(hidden) if give[2] else None, rows, m, n, k, count, CODE[prec], p(base), n, p(dX), n, p(dA), p(dB))
        for got, want in zip((dX, dA, dB), whole):
            assert got is None or same(got, want), give


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 5), (7, 130), (3, 8192), (1100, 520), (2, 40000), (5, 40003)])
def test_norm_without_sum(lrc, prec, rows, n):
    """Rows that the registers hold, and longer ones, whose sum is formed again."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x, r = (torch.randn(rows, n, generator=g, device="cuda").to(DT[prec]) for _ in range(2))
    w = 1 + 0.2 * torch.randn(n, generator=g, device="cuda")
    y, _, rstd = lrc.rms_norm(x, w, residual=r, stats=True)
    codes, scales, _ = lrc.rms_norm_e4m3(x, w, residual=r)
    y2, s2, c2, t2, s3 = torch.empty_like(y), torch.empty_like(rstd), torch.empty_like(codes), torch.empty_like(scales), torch.empty_like(rstd)
    c = CODE[prec]
    lrc._launch(x.device, "lrc_rms_norm", p(x), n, p(r), n, rows, n, c, p(w), 1, 1e-6, None, 0, p(y2), n, c, None, p(s2))
    lrc._launch(x.device, "lrc_rms_norm", p(x), n, p(r), n, rows, n, c, p(w), 1, 1e-6, None, 0, p(c2), n, 4, p(t2), p(s3))
    for got, want in ((y2, y), (s2, rstd), (c2, codes), (t2, scales), (s3, rstd)):
        assert same(got, want)


@pytest.mark.parametrize("prec", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,n", [(3, 7), (40, 1000), (1100, 264), (2, 40003)])
def test_norm_gradient_without_weight_or_its_gradient(lrc, prec, rows, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    h, dy = (torch.randn(rows, n, generator=g, device="cuda").to(DT[prec]) for _ in range(2))
    ones = torch.ones(n, device="cuda")
    rstd = lrc.rms_norm(h, ones, stats=True)[2]
    dx, dw = lrc.rms_norm_backward(dy, h, ones, rstd)
    for weight, dweight in ((ones, None), (None, torch.full_like(dw, 7.0)), (None, None)):
        got = torch.full_like(dx, 7.0)
        lrc._launch(h.device, "lrc_rms_norm_backward", p(dy), n, p(h), n, p(rstd), rows, n, CODE[prec], p(weight), 1, None, 0, p(got), n,
                    p(dweight))
        assert same(got, dx) and (dweight is None or same(dweight, dw))


def test_verification_without_accepted(lrc):
    g = torch.Generator(device="cuda").manual_seed(3)
    for R, D, V in ((3, 4, 1000), (150, 2, 33), (5, 0, 700)):
        L = torch.randn(R, D + 1, V, generator=g, device="cuda") * 3
        d = torch.randint(0, V, (R, D), generator=g, device="cuda")
        u = torch.rand(R, D + 1, generator=g, device="cuda") * 0.3
        want, _ = lrc.verify(L, d, u)
        got = torch.full_like(want, -7)
        lrc._launch(L.device, "lrc_verify", p(L), V, (D + 1) * V, None, 0, 0, R, D, V, 1, p(d) if D else None, p(u), None, None, None, None,
                    p(got), None)
        assert same(got, want)
