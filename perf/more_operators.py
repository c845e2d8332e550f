"""Timed cases of a serving and training step around the compressed projections: the norm in front of them, their product
with 8-bit activations, low-rank adapters of many requests beside them, and the verification of drafted tokens behind.

Four operators of the public Python binding, each with its plain form in elementary torch operations:

  norm      h = x + residual, y = h rsqrt(mean h^2 + eps) w, y as it is or in e4m3 with one scale per row; and its gradient
  q8        Y = t (X8 W4^T + (X8 V diag(s)) U^T): 4-bit weights with rank compensation, e4m3 activations with a scale t per row
  adapter   Y_i = base_i + c_a (X_i A_a^T) B_a^T, a = ids_i: one of N rank-k adapters for each row, or none; and its gradient
  verify    drafted tokens accepted or replaced so that the tokens follow the target's filtered distribution

Sizes are those of the repository's workloads (512 x 256, 8192 x 8192, 65536 x 4096) and generic odd ones.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2, "e4m3": 1}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # magnitudes of codes 0..7; bit 3 is the sign
EPS = 1e-6

MAX_FLOPS = 5.5e11    # the 8192 x 8192 product with 4096 rows
MAX_BYTES = 4.3e8     # a training step of the adapters, 4096 rows of 8192
SHARE = 0.875         # of the draft places that hold a token: one request in four has fewer, any number of them


def listed():
    return [
        # one token: latency
        dict(name="norm_token", op="norm", mode="serve", prec="bf16", wprec="bf16", out="e4m3", residual=True, rows=1, n=8192),
        # a prompt's tokens into 8 bits, in front of the 4-bit product: memory bounds it
        dict(name="norm_prompt", op="norm", mode="serve", prec="bf16", wprec="bf16", out="e4m3", residual=True, rows=4096, n=8192),
        # a training step with odd sizes and binary32 weights
        dict(name="norm_step_ragged", op="norm", mode="step", prec="bf16", wprec="fp32", out="bf16", residual=True, rows=2047, n=5003),
        # one token through a square projection: the weights' bytes bound it
        dict(name="q8_token", op="q8", out="bf16", m=8192, n=8192, k=65, group=128, batch=1),
        # a serving batch through the output head, binary32 logits
        dict(name="q8_head_batch48", op="q8", out="fp32", m=65536, n=4096, k=65, group=128, batch=48),
        # a prompt's tokens: bound by the matrix cores
        dict(name="q8_prompt", op="q8", out="bf16", m=8192, n=8192, k=65, group=128, batch=4096),
        # one token of a small projection: the shortest call
        dict(name="adapter_token_small", op="adapter", mode="serve", prec="fp16", rows=1, m=512, n=256, k=8, count=4),
        # a serving batch, a request's adapter for each row
        dict(name="adapter_batch48", op="adapter", mode="serve", prec="bf16", rows=48, m=8192, n=8192, k=16, count=32),
        # prompts of several requests, sequences of any length
        dict(name="adapter_prompts", op="adapter", mode="serve", prec="bf16", rows=4096, m=8192, n=8192, k=64, count=8),
        # a training step of a few adapters at once
        dict(name="adapter_step", op="adapter", mode="step", prec="bf16", rows=4096, m=8192, n=8192, k=16, count=4),
        # one request with drafts: latency
        dict(name="verify_one", op="verify", prec="fp32", requests=1, drafts=4, vocab=32003, draft_logits=True, masked=0.0),
        # a serving batch over the head's vocabulary
        dict(name="verify_batch48", op="verify", prec="fp32", requests=48, drafts=5, vocab=65536, draft_logits=True, masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd_or_round(rng, x, step):
    """Half of the sizes as drawn (odd ones among them), half rounded to a multiple of step."""
    return x if rng.random() < 0.5 else max(step, x // step * step)


def draw(rng):
    while True:
        op = rng.choice(["norm", "q8", "adapter", "verify"])
        prec = rng.choice(["bf16", "fp16", "fp32"])
        if op == "norm":
            mode = rng.choice(["serve", "serve", "step"])
            c = dict(op=op, mode=mode, prec=prec, wprec=rng.choice([prec, "fp32"]),
                     out=rng.choice([prec, "e4m3"]) if mode == "serve" else prec, residual=rng.random() < 0.7,
                     rows=_log_int(rng, 1, 8192), n=_odd_or_round(rng, _log_int(rng, 256, 16384), 64))
        elif op == "q8":
            m = _odd_or_round(rng, _log_int(rng, 256, 65536), 64)
            n = _odd_or_round(rng, _log_int(rng, 256, 8192), 64)
            # tokens of one sequence, of a serving batch, of prompts
            batch = rng.choice([1, rng.randint(2, 16), rng.randint(17, 64), _log_int(rng, 65, 4096)])
            c = dict(op=op, out=prec, m=m, n=n, k=rng.choice([0, min(_log_int(rng, 8, 128), m, n)]),
                     group=rng.choice([32, 64, 128]), batch=batch)
        elif op == "adapter":
            c = dict(op=op, mode=rng.choice(["serve", "serve", "step"]), prec=prec,
                     rows=rng.choice([1, rng.randint(2, 64), _log_int(rng, 65, 4096)]),
                     m=_odd_or_round(rng, _log_int(rng, 256, 8192), 64), n=_odd_or_round(rng, _log_int(rng, 256, 8192), 64),
                     k=rng.choice([4, 8, 16, 32, 64, 128, rng.randint(1, 128)]), count=_log_int(rng, 1, 64))
        else:
            c = dict(op=op, prec=prec, requests=_log_int(rng, 1, 128), drafts=rng.randint(1, 8),
                     vocab=_odd_or_round(rng, _log_int(rng, 1000, 131072), 64), draft_logits=rng.random() < 0.7,
                     masked=rng.choice([0.0, 0.5, 0.98]))
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return c


# ------------------------------------------------------------------ inputs --

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _gauss(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def _prepare_norm(case, g):
    rows, n, dt = case["rows"], case["n"], DTYPES[case["prec"]]
    # a few channels are much larger than the others, as in a model's residual stream
    channel = 1.0 + 20.0 * (_uniform(g, n) < 0.01).float()
    st = dict(x=_gauss(g, rows, n).to(dt), residual=None, w=(1.0 + 0.1 * _gauss(g, n)).to(DTYPES[case["wprec"]]),
              mode=case["mode"], out=E4M3 if case["out"] == "e4m3" else dt)
    if case["residual"]:
        st["residual"] = (_gauss(g, rows, n) * channel * 3.0).to(dt)
    if case["mode"] == "step":
        st["dy"] = (_gauss(g, rows, n) * 0.1).to(dt)
        st["dsum"] = (_gauss(g, rows, n) * 0.1).to(dt) if case["residual"] else None
    return st


def _prepare_q8(case, g):
    m, n, group, k = case["m"], case["n"], case["group"], case["k"]
    W = _gauss(g, m, n) * ((0.5 + _uniform(g, m, 1)) / math.sqrt(n))
    G = -(-n // group)
    w = torch.nn.functional.pad(W, (0, G * group - n)).view(m, G, group)
    scales = (w.abs().amax(2) / 6).half()
    ratio = (w / scales.float()[:, :, None]).nan_to_num_(0.0)
    mid = torch.tensor([(a + b) / 2 for a, b in zip(E2M1, E2M1[1:])], device="cuda")
    code = torch.bucketize(ratio.abs(), mid) + 8 * torch.signbit(ratio)
    code = code.to(torch.uint8).view(m, G * group)[:, :n]
    code = torch.nn.functional.pad(code, (0, -(-n // 32) * 32 - n))
    factors = None
    if k:
        # the leading singular triplets of what the codes leave: small, slowly decaying
        s = 0.1 * torch.arange(1, k + 1, device="cuda", dtype=torch.float32) ** -0.25
        factors = ((_gauss(g, m, k) / math.sqrt(m)).half(), s.half(), (_gauss(g, n, k) / math.sqrt(n)).half())
    X = _gauss(g, case["batch"], n) * (0.5 + _uniform(g, case["batch"], 1))
    t = X.abs().amax(1) / E4M3_MAX
    return dict(codes=code[:, 0::2] | (code[:, 1::2] << 4), scales=scales, group=group, factors=factors,
                X=(X / t[:, None]).to(E4M3), t=t, out=DTYPES[case["out"]])


def _prepare_adapter(case, g):
    rows, m, n, k, N, dt = case["rows"], case["m"], case["n"], case["k"], case["count"], DTYPES[case["prec"]]
    # requests of a batch, sequences of prompts: an adapter for each, one request in ten without
    starts = torch.ones(rows, device="cuda") if rows <= 64 else (_uniform(g, rows) < max(16.0, rows / 12) ** -1).float()
    sequence = starts.cumsum(0).long()
    which = (_uniform(g, rows + 1) * N).long().clamp_(max=N - 1)
    which = torch.where(_uniform(g, rows + 1) < 0.1, torch.full_like(which, -1), which)
    ids = which[sequence].contiguous()
    st = dict(X=_gauss(g, rows, n).to(dt), A=(_gauss(g, N, k, n) / math.sqrt(n)).to(dt),
              B=(_gauss(g, N, m, k) * (0.3 / math.sqrt(k))).to(dt), ids=ids, scale=0.5 + _uniform(g, N),
              base=_gauss(g, rows, m).to(dt), mode=case["mode"])
    if case["mode"] == "step":
        st["dY"] = (_gauss(g, rows, m) * 0.1).to(dt)
    return st


def _prepare_verify(case, g):
    R, D, V, dt = case["requests"], case["drafts"], case["vocab"], DTYPES[case["prec"]]

    # what requests ask for: one in eight greedy, each filter on in about half of them
    def some(values, off, p):
        return torch.where(_uniform(g, R) < p, values, torch.full_like(values, off))
    st = dict(temperature=some(0.5 + _uniform(g, R), 0.0, 0.875),
              top_k=some((1 + 200 * _uniform(g, R)).long(), 0, 0.5),
              top_p=some(0.5 + 0.49 * _uniform(g, R), 1.0, 0.6),
              min_p=some(0.001 + 0.1 * _uniform(g, R), 0.0, 0.4), u=_uniform(g, R, D + 1))
    logits = _gauss(g, R, D + 1, V) * 2.0 + 6.0 * _uniform(g, R, D + 1, V).pow(64)      # a bulk and a few likely tokens
    if case["masked"]:
        logits.masked_fill_(_uniform(g, R, 1, V) < case["masked"], float("-inf"))
    # the draft model is near the target
    draft = (logits[:, :D] + 0.5 * _gauss(g, R, D, V)).to(dt)
    st["logits"] = logits.to(dt)
    drawn = torch.multinomial(_plain_weights_of(draft, st).view(R * D, V).double(), 1, generator=g).view(R, D)
    # requests with fewer drafts than places
    have = torch.where(_uniform(g, R) < 0.25, (_uniform(g, R) * (D + 1)).long(), torch.full((R,), D, device="cuda"))
    st["drafts"] = drawn.masked_fill(torch.arange(D, device="cuda")[None, :] >= have[:, None], -1)
    st["draft_logits"] = draft if case["draft_logits"] else None
    return st


def prepare(case, seed):
    st = PREPARE[case["op"]](case, _generator(seed))
    st["op"] = case["op"]
    return st


PREPARE = {"norm": _prepare_norm, "q8": _prepare_q8, "adapter": _prepare_adapter, "verify": _prepare_verify}


# --------------------------------------------------------------------- run --

def run(state):
    return _own_run(state) if own else PLAIN[state["op"]](state)


def _own_run(st):
    from paper_2607_12969_amd import lrc
    if st["op"] == "norm":
        if st["mode"] == "step":
            y, h, rstd = lrc.rms_norm(st["x"], st["w"], residual=st["residual"], eps=EPS, stats=True)
            dx, dw = lrc.rms_norm_backward(st["dy"], h, st["w"], rstd, dsum=st["dsum"])
            return {"y": y, "h": h, "dx": dx, "dw": dw}
        if st["out"] == E4M3:
            y, scales, h = lrc.rms_norm_e4m3(st["x"], st["w"], residual=st["residual"], eps=EPS)
            return {"y": y, "scales": scales, "h": h}
        y, h = lrc.rms_norm(st["x"], st["w"], residual=st["residual"], eps=EPS)
        return {"y": y, "h": h}
    if st["op"] == "q8":
        return lrc.q4_apply(st["codes"], st["scales"], st["X"], group=st["group"], factors=st["factors"],
                            out_dtype=st["out"], x_scales=st["t"])
    if st["op"] == "adapter":
        if st["mode"] == "serve":
            return lrc.adapter_apply(st["X"], st["A"], st["B"], st["ids"], scale=st["scale"], base=st["base"])
        Y, hidden = lrc.adapter_apply(st["X"], st["A"], st["B"], st["ids"], scale=st["scale"], base=st["base"], hidden=True)
        dX, dA, dB = lrc.adapter_backward(st["dY"], st["X"], st["A"], st["B"], st["ids"], hidden, scale=st["scale"])
        return {"Y": Y, "dX": dX, "dA": dA, "dB": dB}
    tokens, accepted = lrc.verify(st["logits"], st["drafts"], st["u"], draft_logits=st["draft_logits"],
                                  temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
    return {"tokens": tokens, "accepted": accepted}


# ------------------------------------------------------------- plain forms --

def _plain_norm(st):
    dt = st["x"].dtype
    h = st["x"] if st["residual"] is None else (st["x"].float() + st["residual"].float()).to(dt)
    hf, w = h.float(), st["w"].float()
    rstd = torch.rsqrt(hf.square().mean(1, keepdim=True) + EPS)
    xhat = hf * rstd
    y = xhat * w
    if st["mode"] == "step":
        dy = st["dy"].float()
        wdy = dy * w
        dx = rstd * (wdy - xhat * (wdy * xhat).mean(1, keepdim=True))
        if st["dsum"] is not None:
            dx = dx + st["dsum"].float()
        return {"y": y.to(dt), "h": h, "dx": dx.to(dt), "dw": (dy * xhat).sum(0).to(st["w"].dtype)}
    if st["out"] == E4M3:
        scales = y.abs().amax(1) / E4M3_MAX
        return {"y": (y / scales[:, None]).to(E4M3), "scales": scales, "h": h}
    return {"y": y.to(dt), "h": h}


def _plain_q8(st):
    x = st["X"].float() * st["t"][:, None]
    codes = st["codes"]
    m, n = codes.shape[0], x.shape[1]
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    W = torch.stack((codes & 15, codes >> 4), dim=2).view(m, -1)[:, :n]
    y = x @ (lut[W.int()] * st["scales"].float().repeat_interleave(st["group"], dim=1)[:, :n]).T
    if st["factors"] is not None:
        U, s, V = (f.float() for f in st["factors"])
        y = y + ((x @ V) * s) @ U.T
    return y.to(st["out"])


def _plain_adapter(st):
    # all adapters side by side, a row's own kept
    X, A, B, dt = st["X"].float(), st["A"].float(), st["B"].float(), st["X"].dtype
    N, k, n = A.shape
    m = B.shape[1]
    mine = (st["ids"][:, None] == torch.arange(N, device=X.device)[None, :]).repeat_interleave(k, dim=1)
    scale = st["scale"].repeat_interleave(k)[None, :]
    A, Bt = A.view(N * k, n), B.transpose(1, 2).reshape(N * k, m)
    zero = torch.zeros((), device=X.device)
    h = torch.where(mine, X @ A.T, zero)
    Y = (st["base"].float() + (h * scale) @ Bt).to(dt)
    if st["mode"] == "serve":
        return Y
    dY = st["dY"].float()
    dh = torch.where(mine, (dY @ Bt.T) * scale, zero)
    dB = ((h * scale).T @ dY).view(N, k, m).transpose(1, 2).contiguous()
    return {"Y": Y, "dX": (dh @ A).to(dt), "dA": (dh.T @ X).view(N, k, n).to(dt), "dB": dB.to(dt)}


def _plain_weights_of(logits, st):
    """R x D x V whole weights of the tokens that each request's temperature and filters keep."""
    l = logits.float()
    l = torch.where(l.isnan(), torch.full_like(l, float("-inf")), l)
    V = l.shape[2]
    M = l.amax(2, keepdim=True)
    T = st["temperature"][:, None, None]
    fmin, fmax = torch.finfo(torch.float32).tiny, torch.finfo(torch.float32).max
    c = ((1.0 / T) * 1.4426950408889634).clamp(fmin, fmax)
    # weights as whole multiples of 2^-31: their sums are exact in any order
    w = torch.exp2(torch.where(l == M, torch.zeros_like(l), (l - M) * c))
    q = (w * 2147483648.0).long()
    order = torch.sort(l, dim=2, descending=True, stable=True).indices
    qs = q.gather(2, order)
    before = qs.cumsum(2) - qs
    rank = torch.arange(V, device=l.device)[None, None, :]
    k = st["top_k"][:, None, None]
    k = torch.where((k <= 0) | (k > V), torch.full_like(k, V), k)
    mass = (before + qs).gather(2, (k - 1).expand(-1, l.shape[1], -1))
    p = st["top_p"][:, None, None].double()
    keep = (rank < k) & (~(p < 1) | (before.double() < p * mass.double()) | (rank == 0))
    mp = st["min_p"][:, None, None]
    keep &= ~(mp > 0) | (w.gather(2, order) >= mp) | (rank == 0)
    keep = torch.where(T > 0, keep, rank == 0)
    qs = torch.where(T > 0, qs, torch.full_like(qs, 1 << 31))
    weights = torch.zeros_like(q).scatter_(2, order, torch.where(keep, qs, torch.zeros_like(qs)))
    return torch.where(M == float("-inf"), torch.zeros_like(weights), weights)


def _plain_verify(st):
    drafts, u = st["drafts"], st["u"].double()
    R, D = drafts.shape
    V = st["logits"].shape[2]
    given = (drafts >= 0) & (drafts < V)
    at = drafts.clamp(0, V - 1)[:, :, None]
    P = _plain_weights_of(st["logits"], st)
    Sp = P.sum(2)
    index = torch.arange(V, device=drafts.device)
    if st["draft_logits"] is None:
        Q = (index[None, None, :] == at).long()         # the draft model is sure
    else:
        Q = _plain_weights_of(st["draft_logits"], st)
    Sq = Q.sum(2)
    p, q = P[:, :D].gather(2, at)[:, :, 0].double(), Q.gather(2, at)[:, :, 0].double()
    accept = (u[:, :D] * q) * Sp[:, :D].double() < p * Sq.double()
    # drafts are taken up to the first that is rejected or missing
    count = (accept & given).long().cumprod(1).sum(1)
    row = torch.arange(R, device=drafts.device)
    last = count.clamp(max=D - 1)
    rejected = (count < D) & given[row, last]
    # there the token comes from what the target has above the draft, in units of 2^-52
    Pn, Qn = P[row, count], Q[row, last]
    share = (Pn.double() * (2.0 ** 52 / Sp[row, count].double())[:, None]).nan_to_num_(0.0).long()
    taken = (Qn.double() * (2.0 ** 52 / Sq[row, last].double())[:, None]).nan_to_num_(0.0).long()
    rest = (share - taken).clamp(min=0)
    rest = torch.where((rejected & (rest.sum(1) > 0))[:, None], rest, Pn)
    cs = rest.cumsum(1)
    S = cs[:, -1:]
    t = torch.minimum((u[:, D:] * S.double()).long(), S - 1)
    token = torch.where(cs > t, index[None, :], V).amin(1)
    token = torch.where(S[:, 0] > 0, token, torch.full_like(token, -1))
    place = torch.arange(D + 1, device=drafts.device)[None, :]
    tokens = torch.nn.functional.pad(drafts, (0, 1), value=-1)
    tokens = torch.where(place < count[:, None], tokens, torch.where(place == count[:, None], token[:, None], -1))
    return {"tokens": tokens, "accepted": count}


PLAIN = {"norm": _plain_norm, "q8": _plain_q8, "adapter": _plain_adapter, "verify": _plain_verify}


# ---------------------------------------------------------------- figures --

def work(case):
    op = case["op"]
    if op == "norm":
        e, rows, n, res = BYTES[case["prec"]], case["rows"], case["n"], case["residual"]
        # x (and the residual) in; y and its statistic (and the sum) out
        bytes_ = rows * n * (e * (3 if res else 1) + BYTES[case["out"]]) + 4 * rows + BYTES[case["wprec"]] * n
        if case["mode"] == "step":
            # dy, h, the statistic (and the sum's gradient) in; dx and dw out
            bytes_ += e * rows * n * (4 if res else 3) + 4 * rows + 2 * BYTES[case["wprec"]] * n
        return dict(bytes=bytes_, flops=(14 if case["mode"] == "step" else 5) * rows * n)
    if op == "q8":
        m, n, k, b = case["m"], case["n"], case["k"], case["batch"]
        return dict(bytes=m * -(-n // 2) + 2 * m * -(-n // case["group"]) + 2 * k * (m + n + 1) + b * n + 4 * b
                    + BYTES[case["out"]] * b * m, flops=2 * b * (m * n + k * (m + n)))
    if op == "adapter":
        e, rows, m, n, k = BYTES[case["prec"]], case["rows"], case["m"], case["n"], case["k"]
        N = min(case["count"], rows)
        bytes_ = e * (rows * (n + 2 * m) + N * k * (n + m)) + 8 * rows
        flops = 2 * rows * k * (n + m)
        if case["mode"] == "step":
            # dY, X and the adapters in, dX and the adapters' gradients out
            bytes_ += e * (rows * (m + 2 * n) + (N + case["count"]) * k * (n + m)) + 8 * rows
            flops *= 3
        return dict(bytes=bytes_, flops=flops)
    e, R, D, V = BYTES[case["prec"]], case["requests"], case["drafts"], case["vocab"]
    rows = int(R * (1 + SHARE * D * (2 if case["draft_logits"] else 1)))
    return dict(bytes=rows * e * V + R * (5 * 4 + 4 * (D + 1) + 8 * D + 8 * (D + 2)), flops=8 * rows * V)


# ------------------------------------------------------------------- exact --

def _exact_norm(st):
    x = st["x"].double()
    h = st["x"] if st["residual"] is None else (x + st["residual"].double()).to(st["x"].dtype)
    H = h.double()
    n = H.shape[1]
    norm = torch.sqrt((H * H).sum(1, keepdim=True) / n + EPS)
    y = st["w"].double() * (H / norm)
    if st["mode"] == "step":
        g = st["dy"].double() * st["w"].double()
        along = (g * H).sum(1, keepdim=True) / (n * norm ** 3)
        dx = g / norm - along * H
        if st["dsum"] is not None:
            dx += st["dsum"].double()
        return {"y": y, "h": H, "dx": dx, "dw": torch.einsum("ij,ij->j", st["dy"].double(), H / norm)}
    if st["out"] == E4M3:
        t = y.abs().max(dim=1).values / E4M3_MAX
        return {"y": y / t[:, None], "scales": t, "h": H}
    return {"y": y, "h": H}


def _exact_q8(st):
    X = st["X"].double()
    n, group = X.shape[1], st["group"]
    lut = torch.tensor([(-1) ** (c >> 3) * E2M1[c & 7] for c in range(16)], dtype=torch.float64, device="cuda")
    Y = torch.zeros(X.shape[0], st["codes"].shape[0], dtype=torch.float64, device="cuda")
    step = 2048 // group * group
    for j in range(0, n, step):
        w = min(step, n - j)
        c = st["codes"][:, j // 2:(j + w + 1) // 2].int()
        W = torch.empty(c.shape[0], 2 * c.shape[1], dtype=torch.float64, device="cuda")
        W[:, 0::2], W[:, 1::2] = lut[c % 16], lut[c // 16]
        W = W[:, :w]
        for i in range(0, w, group):
            W[:, i:i + group] *= st["scales"][:, (j + i) // group, None].double()
        Y.addmm_(X[:, j:j + w], W.T)
    if st["factors"] is not None:
        U, s, V = (f.double() for f in st["factors"])
        Y += (X @ (V * s)) @ U.T
    return Y.mul_(st["t"].double()[:, None])


def _exact_adapter(st):
    Y = st["base"].double()
    step = st["mode"] == "step"
    if step:
        dX = torch.zeros(st["X"].shape, dtype=torch.float64, device="cuda")
        dA = torch.zeros(st["A"].shape, dtype=torch.float64, device="cuda")
        dB = torch.zeros(st["B"].shape, dtype=torch.float64, device="cuda")
    for a in range(st["A"].shape[0]):
        rows = torch.nonzero(st["ids"] == a)[:, 0]
        if len(rows) == 0:
            continue
        X, c = st["X"][rows].double(), float(st["scale"][a])
        A, B = st["A"][a].double(), st["B"][a].double()
        T = X @ A.T
        Y[rows] += c * (T @ B.T)
        if step:
            dY = st["dY"][rows].double()
            dT = c * (dY @ B)
            dX[rows] = dT @ A
            dA[a] = dT.T @ X
            dB[a] = c * (dY.T @ T)
    return {"Y": Y, "dX": dX, "dA": dA, "dB": dB} if step else Y


def exact(case, seed):
    if case["op"] == "verify":
        return None         # tokens are choices, not computed numbers
    return {"norm": _exact_norm, "q8": _exact_q8, "adapter": _exact_adapter}[case["op"]](prepare(case, seed))
