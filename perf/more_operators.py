"""The operators at the two ends of a language model's training step, as cases that can be timed and
compared: layer norm and its backward pass with the reduction of the parameters' gradients, the
embedding lookup and its gradient by sorted tokens, distillation from a teacher's top logits.

`own` False: elementary torch operations in 32 bits.  `own` True: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BETA1, BETA2, EPS, N_MICRO = 0.9, 0.999, 1e-8, 8
NORM_EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}


# ---- cases -------------------------------------------------------------------------------------

def listed():
    return [
        # the norm of one token's hidden state, GPT-2-XL's width: nothing but latency
        dict(name="norm one token", op="norm", rows=1, dim=1600, x="f32", y="bf16", pitch=0),
        # a GPT-2-XL-shaped micro-batch of 4096 tokens, residual stream in fp32, bf16 for the products behind
        dict(name="norm 4096x1600", op="norm", rows=4096, dim=1600, x="f32", y="bf16", pitch=0),
        # its backward pass, parameters' gradients folded into their moments
        dict(name="norm_back 4096x1600 folded", op="norm_back", rows=4096, dim=1600, x="bf16", y="bf16", pitch=0, fold=True),
        # Llama-7B's width, a long batch, gradients of the parameters written
        dict(name="norm_back 16384x4096", op="norm_back", rows=16384, dim=4096, x="bf16", y="bf16", pitch=0, fold=False),
        # the tokens that a server has just sampled
        dict(name="embed 7 tokens", op="embed", tokens=7, vocab=50257, dim=1600, table="bf16", out="bf16", scale=1.0, ids="zipf", pad=0.0),
        # a training batch, vectors scaled by the root of their length
        dict(name="embed 16384x4096", op="embed", tokens=16384, vocab=32000, dim=4096, table="bf16", out="bf16", scale=64.0, ids="zipf", pad=0.0),
        # a short batch of a small odd model, in fp32, gradient written, a tenth of the tokens padding
        dict(name="embed_back 131x257", op="embed_back", tokens=131, vocab=1003, dim=257, table="f32", out="f32", scale=1.0, ids="zipf", pad=0.1,
             mode="write"),
        # a GPT-2-XL-shaped micro-batch folded into the moments
        dict(name="embed_back 4096x1600 folded", op="embed_back", tokens=4096, vocab=50257, dim=1600, table="f32", out="bf16", scale=1.0, ids="zipf",
             pad=0.0, mode="fold"),
        # a long Llama-7B-shaped batch, the whole table's gradient written for a norm and a one-pass update
        dict(name="embed_back 32768x4096", op="embed_back", tokens=32768, vocab=32000, dim=4096, table="bf16", out="bf16", scale=64.0, ids="zipf",
             pad=0.05, mode="write"),
        # the answer of one short conversation, teacher's probabilities as served (with their log-sum)
        dict(name="distill 24x32000", op="distill", tokens=24, vocab=32000, top=20, logits="f32", teacher="f32", out="bf16", scale=1.0, lse=True),
        # a GPT-2-XL-shaped micro-batch: odd rows, a quarter of the tokens are prompt and masked, temperature 2
        dict(name="distill 4096x50257", op="distill", tokens=4096, vocab=50257, top=64, logits="bf16", teacher="bf16", out="bf16", scale=0.5, lse=False),
        # a 128 Ki vocabulary in fp32, gradient in bf16 (the dY of the weight-gradient call)
        dict(name="distill 1500x131072", op="distill", tokens=1500, vocab=131072, top=100, logits="f32", teacher="f32", out="bf16", scale=1.0, lse=True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["norm", "norm_back", "embed", "embed_back", "distill"])
    kind = lambda: rng.choice(["bf16", "f32"])  # noqa: E731
    if op == "distill":
        vocab = _log_between(rng, 500, 160_000)
        logits = kind()
        tokens = _log_between(rng, 1, max(2, min(8192, 200_000_000 // vocab)))
        return dict(op=op, tokens=max(1, tokens // (2 if logits == "f32" else 1)), vocab=vocab, top=_log_between(rng, 1, 128), logits=logits,
                    teacher=kind(), out=rng.choice(["bf16", logits]), scale=rng.choice([1.0, 0.5, 0.25]), lse=rng.random() < 0.5)
    dim = _log_between(rng, 24, 8192)
    if rng.random() < 0.6:
        dim = max(8, dim // 8 * 8)                   # widths are multiples of something, mostly
    if op in ("norm", "norm_back"):
        rows = _log_between(rng, 1, max(2, min(65536, 33_000_000 // dim)))
        case = dict(op=op, rows=rows, dim=dim, x=kind(), y=kind(), pitch=rng.choice([0, 0, 0, 8, 3]))
        if op == "norm_back":
            case["fold"] = rng.random() < 0.5
        return case
    tokens = _log_between(rng, 1, max(2, min(65536, 67_000_000 // dim)))
    case = dict(op=op, tokens=tokens, vocab=_log_between(rng, 100, max(101, min(160_000, 130_000_000 // dim))), dim=dim, table=kind(), out=kind(),
                scale=rng.choice([1.0, math.sqrt(dim)]), ids=rng.choice(["zipf", "zipf", "even"]), pad=rng.choice([0.0, 0.0, 0.3]))
    if op == "embed_back":
        case["mode"] = rng.choice(["write", "add", "fold"])
        case["tokens"] = max(1, tokens // 2)
        if case["mode"] == "fold":                   # moments are fp32, two of them
            case["vocab"] = max(100, case["vocab"] // 2)
    return case


def _chances(case):
    """Probability of each token of the vocabulary: by rank, like text, or all alike."""
    rank = torch.arange(case["vocab"], dtype=torch.float64)
    p = 1 / (rank + 2.7) if case["ids"] == "zipf" else torch.ones_like(rank)
    return p / p.sum()


def _live(case):
    """Rows that are answers: a batch of eight sequences whose first quarter is prompt."""
    seq = max(1, case["tokens"] // 8)
    return [t for t in range(case["tokens"]) if t % seq >= seq // 4]


def work(case):
    if case["op"] in ("norm", "norm_back"):
        n, sx, sy = case["rows"] * case["dim"], SIZES[case["x"]], SIZES[case["y"]]
        if case["op"] == "norm":
            return {"bytes": n * (sx + sy) + 8 * case["rows"] + 8 * case["dim"], "flops": 8 * n}
        return {"bytes": n * (2 * sx + sy) + 8 * case["rows"] + case["dim"] * (4 + (32 if case["fold"] else 8)), "flops": 14 * n}
    if case["op"] in ("embed", "embed_back"):
        T, D, V = case["tokens"], case["dim"], case["vocab"]
        seen = float((1 - (1 - _chances(case)) ** (T * (1 - case["pad"]))).sum())   # tokens that occur, on average
        live = T * (1 - case["pad"])
        if case["op"] == "embed":
            return {"bytes": int(seen * D * SIZES[case["table"]] + T * D * SIZES[case["out"]] + 8 * T), "flops": int(live * D)}
        size = SIZES[case["table"]]
        moved = {"write": V * D * size, "add": 2 * seen * D * size, "fold": 16 * seen * D}[case["mode"]]
        return {"bytes": int(live * D * SIZES[case["out"]] + moved + 8 * T), "flops": int((live + 5 * seen) * D)}
    live = len(_live(case))
    entry = 8 + SIZES[case["teacher"]]
    return {"bytes": live * (case["vocab"] * SIZES[case["logits"]] + case["top"] * entry) + case["tokens"] * (case["vocab"] * SIZES[case["out"]] + 12),
            "flops": 9 * live * case["vocab"]}


# ---- inputs ------------------------------------------------------------------------------------

def _rows(rows, cols, pitch, dtype):
    """[rows, cols] whose rows lie `pitch` elements further apart than they are long."""
    return torch.empty(rows, cols + pitch, device="cuda", dtype=dtype)[:, :cols]


def _prepare_norm(case, gen):
    R, D = case["rows"], case["dim"]
    xt, yt = DTYPES[case["x"]], DTYPES[case["y"]]
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    s = {"case": case, "x": _rows(R, D, case["pitch"], xt), "weight": 1 + 0.1 * normal(D), "bias": 0.1 * normal(D)}
    offset = 0.3 * normal(D)
    offset[::97] *= 30                               # a few channels of a residual stream are large in every token
    s["x"].copy_(normal(R, D).mul_(1 + 0.5 * normal(R, 1).abs()).add_(offset))
    if case["op"] == "norm":
        s["y"] = _rows(R, D, case["pitch"], yt)
        s["mean"], s["rstd"] = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
        return s
    s["mean"], s["rstd"] = _norm_statistics(s["x"].double(), NORM_EPS)
    s["mean"], s["rstd"] = s["mean"].float(), s["rstd"].float()
    s["dy"] = _rows(R, D, case["pitch"], yt)
    s["dy"].copy_(normal(R, D).mul_(1e-3).add_(2e-4 * normal(D)))
    s["dx"] = _rows(R, D, case["pitch"], xt)
    if case["fold"]:
        s["m"] = [1e-3 * normal(D) for _ in range(2)]
        s["v"] = [1e-6 * normal(D).square() for _ in range(2)]
    else:
        s["dweight"], s["dbias"] = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    return s


def _norm_statistics(x, eps):
    mean = x.mean(1)
    return mean, 1 / torch.sqrt((x - mean[:, None]).square().mean(1) + eps)


def _prepare_embed(case, gen):
    T, V, D = case["tokens"], case["vocab"], case["dim"]
    reached = _chances(case).cumsum(0).cuda()
    names = torch.randperm(V, device="cuda", generator=gen)      # rank -> token
    drawn = torch.rand(T, device="cuda", generator=gen, dtype=torch.float64)
    ids = names[torch.searchsorted(reached, drawn).clamp(max=V - 1)]
    if case["pad"]:
        ids[torch.rand(T, device="cuda", generator=gen) < case["pad"]] = -1
    s = {"case": case, "ids": ids}
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    if case["op"] == "embed":
        s["table"] = normal(V, D).mul_(0.02).to(DTYPES[case["table"]])
        s["out"] = torch.empty(T, D, device="cuda", dtype=DTYPES[case["out"]])
        return s
    s["dy"] = normal(T, D).mul_(1e-3).to(DTYPES[case["out"]])
    if case["mode"] == "fold":
        s["m"] = normal(V, D).mul_(1e-5)
        s["v"] = normal(V, D).square_().mul_(1e-10)
    elif case["mode"] == "add":
        s["grad"] = normal(V, D).mul_(1e-3).to(DTYPES[case["table"]])
    else:
        s["grad"] = torch.empty(V, D, device="cuda", dtype=DTYPES[case["table"]])
    return s


def _prepare_distill(case, gen):
    T, V, K = case["tokens"], case["vocab"], case["top"]
    logits = torch.randn(T, V, device="cuda", generator=gen, dtype=DTYPES[case["logits"]]).mul_(2)
    ids = torch.empty(T, K, device="cuda", dtype=torch.int64)
    at = 0
    for rows in torch.empty(T, 0).split(max(1, 4_000_000 // V)):  # K different tokens of each row
        n = rows.shape[0]
        ids[at:at + n] = torch.rand(n, V, device="cuda", generator=gen).topk(K, 1).indices
        at += n
    # a teacher's largest logits fall off from some 8 above the rest; the student mostly agrees
    teacher = 14 - 1.5 * torch.arange(1, K + 1, device="cuda").log()[None, :] + torch.randn(T, K, device="cuda", generator=gen)
    teacher = teacher.sort(1, descending=True).values.to(DTYPES[case["teacher"]])
    logits.scatter_(1, ids, (teacher.float() - 4 + torch.randn(T, K, device="cuda", generator=gen)).to(logits.dtype))
    live = torch.tensor(_live(case), device="cuda")
    s = {"case": case, "logits": logits, "ids": ids, "teacher": teacher}
    s["weights"] = torch.zeros(T, device="cuda").index_fill_(0, live, 1.0 / live.numel())
    # what the teacher's other tokens add to its log-sum: a few per cent of the mass
    s["lse"] = None
    if case["lse"]:
        rest = 1 + 0.1 * torch.rand(T, device="cuda", generator=gen)
        s["lse"] = torch.logsumexp(teacher.float() * case["scale"], 1) + torch.log(rest)
    s["dlogits"] = torch.empty(T, V, dtype=DTYPES[case["out"]], device="cuda")
    s["stats"], s["loss"] = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) & 0x7FFFFFFF)
    make = {"norm": _prepare_norm, "norm_back": _prepare_norm, "embed": _prepare_embed, "embed_back": _prepare_embed, "distill": _prepare_distill}
    s = make[case["op"]](case, gen)
    if own:  # the context, which a training program makes once; a mini-batch of N_MICRO folds has begun
        import paper_2305_19982_b200 as adama
        s["opt"] = adama.AdamA(BETA1, BETA2, EPS)
        s["opt"].begin_minibatch(N_MICRO)
    return s


# ---- the library's calls -----------------------------------------------------------------------

def _own_norm(s):
    s["opt"].layer_norm(s["x"], s["weight"], s["bias"], s["y"], mean=s["mean"], rstd=s["rstd"], eps=NORM_EPS)
    return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}


def _own_norm_back(s):
    given = (s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"])
    if s["case"]["fold"]:
        s["opt"].layer_norm_backward_fold(*given, s["m"][0], s["v"][0], s["m"][1], s["v"][1])
        return {"dx": s["dx"], "m": s["m"], "v": s["v"]}
    s["opt"].layer_norm_backward(*given, s["dweight"], s["dbias"])
    return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}


def _own_embed(s):
    s["opt"].embedding(s["ids"], s["table"], s["out"], scale=s["case"]["scale"])
    return s["out"]


def _own_embed_back(s):
    case = s["case"]
    if case["mode"] == "fold":
        s["opt"].embedding_grad_fold(s["ids"], s["dy"], s["m"], s["v"], scale=case["scale"])
        return {"m": s["m"], "v": s["v"]}
    s["opt"].embedding_grad(s["ids"], s["dy"], s["grad"], scale=case["scale"], accumulate=case["mode"] == "add")
    return s["grad"]


def _own_distill(s):
    s["opt"].distill_loss(s["logits"], s["teacher"], s["ids"], s["weights"], s["dlogits"], s["stats"], teacher_lse=s["lse"], loss=s["loss"],
                          logit_scale=s["case"]["scale"])
    return {"dlogits": s["dlogits"], "stats": s["stats"], "loss": s["loss"]}


# ---- the plain forms: elementary operations in 32 bits -------------------------------------------

def _plain_norm(s):
    x = s["x"].float()
    mean, rstd = _norm_statistics(x, NORM_EPS)
    y = (x - mean[:, None]) * rstd[:, None] * s["weight"] + s["bias"]
    return {"y": y.to(DTYPES[s["case"]["y"]]), "mean": mean, "rstd": rstd}


def _fold(m, v, g):
    m.add_(g * ((1 - BETA1) / N_MICRO))
    v.add_(g * ((1 - BETA2) / N_MICRO ** 2) * g)


def _plain_norm_back(s):
    dy = s["dy"].float()
    xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"]
    along = g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)
    out = {"dx": (along * s["rstd"][:, None]).to(DTYPES[s["case"]["x"]])}
    sums = ((dy * xhat).sum(0), dy.sum(0))
    if not s["case"]["fold"]:
        return {**out, "dweight": sums[0], "dbias": sums[1]}
    for m, v, total in zip(s["m"], s["v"], sums):
        _fold(m, v, total)
    return {**out, "m": s["m"], "v": s["v"]}


def _plain_embed(s):
    rows = s["table"][s["ids"].clamp(min=0)].float() * s["case"]["scale"]
    return torch.where(s["ids"][:, None] >= 0, rows, 0.0).to(DTYPES[s["case"]["out"]])


def _plain_embed_back(s):
    case = s["case"]
    live = s["ids"] >= 0
    g = torch.zeros(case["vocab"], case["dim"], device="cuda")
    g.index_add_(0, s["ids"].clamp(min=0), torch.where(live[:, None], s["dy"].float(), 0.0))
    g = g * case["scale"]
    if case["mode"] == "fold":
        _fold(s["m"], s["v"], g)
        return {"m": s["m"], "v": s["v"]}
    if case["mode"] == "add":
        s["grad"] = (s["grad"].float() + g).to(DTYPES[case["table"]])
        return s["grad"]
    return g.to(DTYPES[case["table"]])


def _plain_distill(s):
    case, scale, wt = s["case"], s["case"]["scale"], s["weights"]
    live = wt != 0
    t = s["teacher"].float() * scale
    top = t.amax(1, keepdim=True)
    logp = t - top - torch.log(torch.exp(t - top).sum(1, keepdim=True)) if s["lse"] is None else t - s["lse"][:, None]
    p = torch.exp(logp)
    mass = p.sum(1)
    z = s["logits"].float() * scale
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    logq = z.gather(1, s["ids"]) - torch.log(total)
    cross = -(p * logq).sum(1)
    kl = (p * logp).sum(1) + cross
    terms = torch.stack([kl, cross, torch.exp(logq).sum(1), mass])
    unit = torch.where(live, wt * scale, 0.0)
    grad = e * ((unit * mass)[:, None] / total)
    grad.scatter_add_(1, s["ids"], -p * unit[:, None])
    return {"dlogits": grad.to(DTYPES[case["out"]]), "stats": torch.where(live, terms * wt, 0.0).sum(1), "loss": torch.where(live, kl, 0.0)}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _own_norm, "norm_back": _own_norm_back, "embed": _own_embed, "embed_back": _own_embed_back, "distill": _own_distill}[op](s)
    return {"norm": _plain_norm, "norm_back": _plain_norm_back, "embed": _plain_embed, "embed_back": _plain_embed_back,
            "distill": _plain_distill}[op](s)


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _folded(s, name, g):
    """Moment `name` after g has been folded; the call's coefficients are 32-bit numbers by definition."""
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    if name == "m":
        return f32((1 - BETA1) / N_MICRO) * g
    return f32((1 - BETA2) / N_MICRO ** 2) * g ** 2


def _exact_norm(s, case):
    x = s["x"].double()
    if case["op"] == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + NORM_EPS) ** -0.5
        return {"y": torch.addcmul(s["bias"].double(), (x - mean[:, None]).mul_(rstd[:, None]), s["weight"].double()), "mean": mean, "rstd": rstd}
    rstd, D = s["rstd"].double()[:, None], case["dim"]
    xhat = (x - s["mean"].double()[:, None]) * rstd
    dy = s["dy"].double()
    w = s["weight"].double()
    # dx = rstd*(I - 11'/D - xhat xhat'/D) (w*dy)
    dx = w * dy
    dx = (dx - (dy @ w)[:, None] / D - xhat * torch.einsum("rd,rd,d->r", dy, xhat, w)[:, None] / D) * rstd
    dweight, dbias = torch.einsum("rd,rd->d", dy, xhat), torch.einsum("rd->d", dy)
    if not case["fold"]:
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    return {"dx": dx, **{k: [old.double() + _folded(s, k, g) for old, g in zip(s[k], (dweight, dbias))] for k in ("m", "v")}}


def _exact_embed(s, case):
    ids = s["ids"]
    if case["op"] == "embed":
        padded = torch.cat([s["table"].double() * case["scale"], torch.zeros(1, case["dim"], device="cuda", dtype=torch.float64)])
        return padded[torch.where(ids < 0, case["vocab"], ids)]
    order = torch.argsort(ids, stable=True)[int((ids < 0).sum()):]    # equal tokens side by side, padding left out
    g = torch.zeros(case["vocab"], case["dim"], device="cuda", dtype=torch.float64)
    if order.numel():
        tokens, counts = torch.unique_consecutive(ids[order], return_counts=True)
        g[tokens] = torch.segment_reduce(s["dy"][order].double(), "sum", lengths=counts, axis=0)
    g *= case["scale"]
    if case["mode"] == "fold":
        return {k: s[k].double() + _folded(s, k, g) for k in ("m", "v")}
    return s["grad"].double() + g if case["mode"] == "add" else g


def _exact_distill(s, case):
    scale, at, parts = case["scale"], 0, []
    for x in s["logits"].split(max(1, 20_000_000 // case["vocab"])):
        rows = slice(at, at + x.shape[0])
        at += x.shape[0]
        logq = torch.log_softmax(x.double() * scale, 1)
        t = s["teacher"][rows].double() * scale
        logp = torch.log_softmax(t, 1) if s["lse"] is None else t - s["lse"][rows].double()[:, None]
        p, wt, ids = logp.exp(), s["weights"][rows].double(), s["ids"][rows]
        mass, at_top = p.sum(1), logq.gather(1, ids)
        kl = (p * (logp - at_top)).sum(1)
        grad = logq.exp_().mul_((wt * scale * mass)[:, None])
        for i in range(case["top"]):
            grad[torch.arange(len(ids), device="cuda"), ids[:, i]] -= wt * scale * p[:, i]
        terms = torch.stack([kl, -(p * at_top).sum(1), at_top.exp().sum(1), mass])
        parts.append((grad, (terms * wt).sum(1), torch.where(wt != 0, kl, 0.0)))
    return {"dlogits": torch.cat([x[0] for x in parts]), "stats": sum(x[1] for x in parts), "loss": torch.cat([x[2] for x in parts])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_back": _exact_norm, "embed": _exact_embed, "embed_back": _exact_embed, "distill": _exact_distill}[case["op"]](s, case)
