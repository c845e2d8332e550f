"""Timed cases of the compressed output head: 4-bit weights with rank compensation, the draw from its logits, and
the loss that fits it to an uncompressed teacher.

Four operators of the public Python binding, each with its plain form in elementary torch operations:

  quantize  W (m x n) -> 4-bit E2M1 codes with one scale per `group` weights of a row, and the values they stand for
  q4        Y = X W4^T + (X V diag(s)) U^T, W4 the weights of stored codes and scales, U, s, V a rank-k compensation
  sample    one token per row of logits, by temperature, top-k, top-p, min-p and a given uniform number
  distill   T^2 KL(teacher || student) per row from the teacher's top logits, and its gradient by the student's logits

Sizes are those of the repository's workloads (512 x 256, 8192 x 8192, 65536 x 4096) and generic odd ones.
"""
import math

import torch

own = False

DTYPES = {"fp64": torch.float64, "fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp64": 8, "fp32": 4, "fp16": 2, "bf16": 2}

MAX_FLOPS = 5.5e11    # the 8192 x 8192 product with 4096 rows
MAX_BYTES = 1.6e9     # the 65536 x 4096 binary32 quantization with its values

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # magnitudes of codes 0..7; bit 3 is the sign
STEPS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def listed():
    return [
        # one token through a small projection: the shortest call, all latency
        dict(name="q4_token_small", op="q4", prec="fp16", out="fp16", m=512, n=256, k=21, group=32, batch=1),
        # one token through a square projection: the weights' bytes bound it
        dict(name="q4_token_square", op="q4", prec="bf16", out="bf16", m=8192, n=8192, k=65, group=128, batch=1),
        # a few sequences, odd sizes, binary32 activations, no compensation
        dict(name="q4_ragged_fp32", op="q4", prec="fp32", out="fp32", m=5003, n=4099, k=0, group=64, batch=7),
        # a serving batch through the output head, binary32 logits
        dict(name="q4_head_batch48", op="q4", prec="fp16", out="fp32", m=65536, n=4096, k=65, group=128, batch=48),
        # a prompt's tokens: bound by the matrix cores
        dict(name="q4_prompt", op="q4", prec="bf16", out="bf16", m=8192, n=8192, k=65, group=128, batch=4096),
        # the head's weights to 4 bits, once per model
        dict(name="quantize_head", op="quantize", prec="fp32", scale="fp16", m=65536, n=4096, group=128),
        # a small projection with odd rows and a last group that is not full
        dict(name="quantize_ragged", op="quantize", prec="bf16", scale="fp32", m=1021, n=2051, group=32),
        # one sequence: latency
        dict(name="sample_one", op="sample", prec="fp32", rows=1, vocab=32003, masked=0.0),
        # a serving batch over the head's vocabulary
        dict(name="sample_batch48", op="sample", prec="fp32", rows=48, vocab=65536, masked=0.0),
        # many sequences, odd vocabulary, half of it forbidden by a grammar
        dict(name="sample_ragged", op="sample", prec="bf16", rows=256, vocab=131071, masked=0.5),
        # a small step, odd sizes, renormalized teacher, loss first and its gradient later
        dict(name="distill_ragged", op="distill", prec="fp32", mode="split", rows=509, vocab=10007, top=17, tail=False,
             temperature=2.0),
        # a training step over the head's vocabulary with the teacher's remaining mass in one class
        dict(name="distill_step", op="distill", prec="bf16", mode="step", rows=4096, vocab=65536, top=64, tail=True,
             temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd_or_round(rng, x, step):
    """Half of the sizes as drawn (odd ones among them), half rounded to a multiple of step."""
    return x if rng.random() < 0.5 else max(step, x // step * step)


def draw(rng):
    while True:
        x = rng.random()
        if x < 5 / 12:
            prec = rng.choice(["fp16", "bf16", "fp32"])
            m = _odd_or_round(rng, _log_int(rng, 256, 65536), 64)
            n = _odd_or_round(rng, _log_int(rng, 256, 8192), 64)
            # tokens of one sequence, of a serving batch, of prompts
            batch = rng.choice([1, rng.randint(2, 16), rng.randint(17, 64), _log_int(rng, 65, 4096)])
            c = dict(op="q4", prec=prec, out=rng.choice([prec, "fp32"]), m=m, n=n,
                     k=rng.choice([0, min(_log_int(rng, 8, 128), m, n)]), group=rng.choice([32, 64, 128]), batch=batch)
        elif x < 7 / 12:
            c = dict(op="quantize", prec=rng.choice(["fp32", "fp16", "bf16", "fp64"]), scale=rng.choice(["fp16", "fp32"]),
                     m=_odd_or_round(rng, _log_int(rng, 256, 65536), 64),
                     n=_odd_or_round(rng, _log_int(rng, 256, 8192), 64), group=rng.choice([32, 64, 128]))
        elif x < 10 / 12:
            c = dict(op="sample", prec=rng.choice(["fp32", "fp16", "bf16"]), rows=_log_int(rng, 1, 256),
                     vocab=_odd_or_round(rng, _log_int(rng, 1000, 131072), 64), masked=rng.choice([0.0, 0.5, 0.98]))
        else:
            c = dict(op="distill", prec=rng.choice(["fp32", "fp16", "bf16"]), mode=rng.choice(["step", "split", "eval"]),
                     rows=_odd_or_round(rng, _log_int(rng, 16, 4096), 16),
                     vocab=_odd_or_round(rng, _log_int(rng, 1000, 131072), 64), top=_log_int(rng, 4, 256),
                     tail=rng.random() < 0.5, temperature=rng.choice([1.0, 2.0, 4.0]))
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return c


# ------------------------------------------------------------------ inputs --

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _gauss(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    g = _generator(seed)
    dt = DTYPES[case["prec"]]
    op = case["op"]
    if op in ("q4", "quantize"):
        m, n, group = case["m"], case["n"], case["group"]
        # rows of different size, normal weights
        W = _gauss(g, m, n) * ((0.5 + _uniform(g, m, 1)) / math.sqrt(n))
        if op == "quantize":
            return dict(op=op, W=W.to(dt), group=group, scale=DTYPES[case["scale"]])
        codes, scales, _ = _plain_quantize(W, group, torch.float16)
        factors = None
        if case["k"]:
            # the leading singular triplets of what the codes leave: small, slowly decaying
            k = case["k"]
            s = 0.1 * torch.arange(1, k + 1, device="cuda", dtype=torch.float32) ** -0.25
            factors = ((_gauss(g, m, k) / math.sqrt(m)).half(), s.half(), (_gauss(g, n, k) / math.sqrt(n)).half())
        return dict(op=op, codes=codes, scales=scales, group=group, factors=factors,
                    X=_gauss(g, case["batch"], n).to(dt), out=DTYPES[case["out"]])
    if op == "sample":
        rows, V = case["rows"], case["vocab"]
        logits = _gauss(g, rows, V) * 2.0 + 6.0 * _uniform(g, rows, V).pow(64)      # a bulk and a few likely tokens
        if case["masked"]:
            logits.masked_fill_(_uniform(g, rows, V) < case["masked"], float("-inf"))
        # what requests ask for: one in eight greedy, each filter on in about half of them
        def some(values, off, p):
            return torch.where(_uniform(g, rows) < p, values, torch.full_like(values, off))
        return dict(op=op, logits=logits.to(dt), u=_uniform(g, rows),
                    temperature=some(0.5 + _uniform(g, rows), 0.0, 0.875),
                    top_k=some((1 + 200 * _uniform(g, rows)).long(), 0, 0.5),
                    top_p=some(0.5 + 0.49 * _uniform(g, rows), 1.0, 0.6),
                    min_p=some(0.001 + 0.1 * _uniform(g, rows), 0.0, 0.4))
    rows, V, K, T = case["rows"], case["vocab"], case["top"], case["temperature"]
    teacher = _gauss(g, rows, V).mul_(2.5)
    student = _gauss(g, rows, V).mul_(0.5).add_(teacher)
    top, ids = torch.topk(teacher, K, dim=1)
    lse = torch.logsumexp(teacher / T, dim=1) if case["tail"] else None
    del teacher
    # rows that know fewer tokens than K, and padding tokens that do not count
    known = torch.where(_uniform(g, rows) < 0.25, (1 + K * _uniform(g, rows)).long(), torch.full((rows,), K, device="cuda"))
    ids = ids.masked_fill(torch.arange(K, device="cuda")[None, :] >= known[:, None], -1)
    weight = (_uniform(g, rows) < 0.9).float()
    # a mean over the counted tokens; binary16 gradients come with a loss scale, as they do in training
    weight *= (65536.0 if dt == torch.float16 else 1.0) / weight.sum().clamp(min=1.0)
    return dict(op=op, mode=case["mode"], logits=student.to(dt), ids=ids, top=top, lse=lse, weight=weight, T=T,
                dloss=0.5 + _uniform(g, rows))


# --------------------------------------------------------------------- run --

def run(state):
    return _own_run(state) if own else _plain_run(state)


def _own_run(st):
    from paper_2607_12969_amd import lrc
    if st["op"] == "quantize":
        codes, scales, values = lrc.q4_quantize(st["W"], group=st["group"], scale_dtype=st["scale"], values=True)
        return {"scales": scales, "values": values}
    if st["op"] == "q4":
        return lrc.q4_apply(st["codes"], st["scales"], st["X"], group=st["group"], factors=st["factors"],
                            out_dtype=st["out"])
    if st["op"] == "sample":
        return lrc.sample(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                          min_p=st["min_p"])
    kw = dict(temperature=st["T"], teacher_lse=st["lse"], weight=st["weight"])
    if st["mode"] == "step":
        loss, grad = lrc.distill(st["logits"], st["ids"], st["top"], **kw)
        return {"loss": loss, "grad": grad}
    loss, stats = lrc.distill_forward(st["logits"], st["ids"], st["top"], **kw)
    if st["mode"] == "eval":
        return {"loss": loss}
    return {"loss": loss, "grad": lrc.distill_backward(st["logits"], st["ids"], st["top"], stats, dloss=st["dloss"], **kw)}


# ------------------------------------------------------------- plain forms --

def _plain_quantize(W, group, scale_dtype):
    m, n = W.shape
    G = -(-n // group)
    w = torch.nn.functional.pad(W if W.dtype == torch.float64 else W.float(), (0, G * group - n)).view(m, G, group)
    scales = (w.abs().amax(2) / 6).to(scale_dtype)
    sc = scales.to(w.dtype)[:, :, None]
    a = (w.abs() / sc).nan_to_num_(0.0)                 # 0 / 0: a group of zeros
    code = torch.zeros(a.shape, dtype=torch.uint8, device=W.device)
    for t, even_up in STEPS:                            # nearest value, ties to the even code
        code += (a >= t) if even_up else (a > t)
    values = torch.tensor(E2M1, device=W.device, dtype=w.dtype)[code.int()] * sc
    neg = torch.signbit(w)
    values = torch.where(neg, -values, values).view(m, G * group)[:, :n].to(W.dtype)
    code += neg.to(torch.uint8) * 8
    code = code.view(m, G * group)[:, :n]
    code = torch.nn.functional.pad(code, (0, -(-n // 32) * 32 - n))
    return code[:, 0::2] | (code[:, 1::2] << 4), scales, values.contiguous()


def _plain_weights(codes, scales, group, n):
    m = codes.shape[0]
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    W = torch.stack((codes & 15, codes >> 4), dim=2).view(m, -1)[:, :n]
    return lut[W.int()] * scales.float().repeat_interleave(group, dim=1)[:, :n]


def _plain_sample(st):
    l = st["logits"].float()
    l = torch.where(l.isnan(), torch.full_like(l, float("-inf")), l)
    rows, V = l.shape
    M = l.amax(1, keepdim=True)
    T = st["temperature"][:, None]
    fmin, fmax = torch.finfo(torch.float32).tiny, torch.finfo(torch.float32).max
    c = ((1.0 / T) * 1.4426950408889634).clamp(fmin, fmax)
    # weights as whole multiples of 2^-31: their sums are exact in any order
    w = torch.exp2(torch.where(l == M, torch.zeros_like(l), (l - M) * c))
    q = (w * 2147483648.0).long()
    order = torch.sort(l, dim=1, descending=True, stable=True).indices
    qs = q.gather(1, order)
    before = qs.cumsum(1) - qs
    rank = torch.arange(V, device=l.device)[None, :]
    k = st["top_k"][:, None]
    k = torch.where((k <= 0) | (k > V), torch.full_like(k, V), k)
    mass = (before + qs).gather(1, k - 1)
    p = st["top_p"][:, None].double()
    keep = (rank < k) & (~(p < 1) | (before.double() < p * mass.double()) | (rank == 0))
    mp = st["min_p"][:, None]
    keep &= ~(mp > 0) | (w.gather(1, order) >= mp) | (rank == 0)
    kept = torch.zeros_like(q).scatter_(1, order, torch.where(keep, qs, torch.zeros_like(qs)))
    cs = kept.cumsum(1)
    S = cs[:, -1:]
    t = torch.minimum((st["u"][:, None].double() * S.double()).long(), S - 1)
    index = torch.arange(V, device=l.device)[None, :]
    token = torch.where(cs > t, index, V).amin(1)
    greedy = torch.where(l == M, index, V).amin(1)
    token = torch.where(T[:, 0] > 0, token, greedy)
    return torch.where(M[:, 0] == float("-inf"), torch.full_like(token, -1), token)


def _plain_distill(st, grad):
    z, T = st["logits"].float(), st["T"]
    e = ((z - z.amax(1, keepdim=True)) / T).exp()
    S = e.sum(1, keepdim=True)
    valid = st["ids"] >= 0
    ids = st["ids"].clamp(min=0)
    tl = torch.where(valid, st["top"].float() / T, torch.full_like(st["top"], float("-inf")))
    lse = st["lse"][:, None] if st["lse"] is not None else torch.logsumexp(tl, dim=1, keepdim=True)
    p = torch.where(valid, (tl - lse).exp(), torch.zeros_like(tl))
    logq = ((z.gather(1, ids) - z.amax(1, keepdim=True)) / T) - S.log()
    kl = torch.where(p > 0, p * (tl - lse - logq), torch.zeros_like(p)).sum(1)
    g = e / S
    if st["lse"] is not None:
        top = torch.zeros(z.shape[0], z.shape[1] + 1, dtype=torch.bool, device=z.device)
        top = top.scatter_(1, torch.where(valid, ids, z.shape[1]), True)[:, :-1]
        Q = torch.where(top, torch.zeros_like(g), g).sum(1, keepdim=True)
        r = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        kl = kl + torch.where(r > 0, r * (r.log() - Q.log()), torch.zeros_like(r))[:, 0]
        g = torch.where(top, g, g * (1 - r / Q))
    loss = st["weight"] * T * T * kl
    if not grad:
        return loss, None
    g.scatter_add_(1, ids, -p)
    scale = st["weight"] * T * (st["dloss"] if st["mode"] == "split" else 1.0)
    return loss, (g * scale[:, None]).to(st["logits"].dtype)


def _plain_run(st):
    if st["op"] == "quantize":
        _, scales, values = _plain_quantize(st["W"], st["group"], st["scale"])
        return {"scales": scales, "values": values}
    if st["op"] == "q4":
        x = st["X"].float()
        y = x @ _plain_weights(st["codes"], st["scales"], st["group"], x.shape[1]).T
        if st["factors"] is not None:
            U, s, V = (f.float() for f in st["factors"])
            y = y + ((x @ V) * s) @ U.T
        return y.to(st["out"])
    if st["op"] == "sample":
        return _plain_sample(st)
    loss, grad = _plain_distill(st, st["mode"] != "eval")
    return {"loss": loss} if st["mode"] == "eval" else {"loss": loss, "grad": grad}


# ---------------------------------------------------------------- figures --

def work(case):
    op, e = case["op"], BYTES[case["prec"]]
    if op in ("q4", "quantize"):
        m, n = case["m"], case["n"]
        codes, groups = m * -(-n // 2), m * -(-n // case["group"])
        if op == "quantize":
            # weights in; codes, scales and values out
            return dict(bytes=2 * e * m * n + codes + BYTES[case["scale"]] * groups, flops=4 * m * n)
        k, b = case["k"], case["batch"]
        return dict(bytes=codes + 2 * groups + 2 * k * (m + n + 1) + e * b * n + BYTES[case["out"]] * b * m,
                    flops=2 * b * (m * n + k * (m + n)))
    if op == "sample":
        return dict(bytes=case["rows"] * (e * case["vocab"] + 5 * 4 + 4 + 8), flops=8 * case["rows"] * case["vocab"])
    N, V, K = case["rows"], case["vocab"], case["top"]
    passes = {"eval": 1, "step": 2, "split": 3}[case["mode"]]     # split: the logits are read by both calls
    return dict(bytes=passes * e * N * V + N * (12 * K + 8), flops=(5 if case["mode"] == "eval" else 9) * N * V)


# ------------------------------------------------------------------- exact --

def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        W = st["W"].double()
        m, n = W.shape
        group = st["group"]
        out, scales = torch.empty_like(W), torch.empty(m, -(-n // group), dtype=torch.float64, device="cuda")
        grid = torch.tensor([-v for v in E2M1[:0:-1]] + list(E2M1), dtype=torch.float64, device="cuda")
        mid = (grid[1:] + grid[:-1]) / 2
        for j in range(scales.shape[1]):
            w = W[:, j * group:(j + 1) * group]
            sc = (w.abs().amax(1) / 6).to(st["scale"]).double()
            ratio = w / torch.where(sc > 0, sc, torch.ones_like(sc))[:, None]
            out[:, j * group:(j + 1) * group] = grid[torch.bucketize(ratio, mid)] * sc[:, None]
            scales[:, j] = sc
        return {"scales": scales, "values": out}
    if op == "q4":
        X = st["X"].double()
        group, n = st["group"], X.shape[1]
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
        return Y
    if op == "sample":
        return None         # a token is a choice, not a computed number
    z, T, w = st["logits"].double() / st["T"], st["T"], st["weight"].double()
    logq = torch.log_softmax(z, dim=1)
    valid = st["ids"] >= 0
    ids = st["ids"].clamp(min=0)
    tl = (st["top"].double() / T).masked_fill(~valid, float("-inf"))
    if st["lse"] is None:
        p = torch.softmax(tl, dim=1)
        logp = torch.log_softmax(tl, dim=1)
    else:
        logp = tl - st["lse"].double()[:, None]
        p = logp.exp()
    kl = (p * (logp - logq.gather(1, ids))).masked_fill(~valid, 0.0).sum(1)
    t = torch.zeros_like(z).scatter_add_(1, ids, p)
    q = logq.exp_()
    if st["lse"] is not None:
        # the rest of both distributions is one more class
        rest = q.clone()
        rest[torch.arange(len(ids), device="cuda")[:, None].expand_as(ids)[valid], ids[valid]] = 0.0
        Q, r = rest.sum(1), (1 - p.sum(1)).clamp(min=0)
        kl += torch.where(r > 0, r * (r / Q).log(), torch.zeros_like(r))
        t += rest.mul_((r / Q)[:, None])
    loss = w * T * T * kl
    if st["mode"] == "eval":
        return {"loss": loss}
    up = st["dloss"].double() if st["mode"] == "split" else torch.ones_like(w)
    return {"loss": loss, "grad": q.sub_(t).mul_((w * T * up)[:, None])}
