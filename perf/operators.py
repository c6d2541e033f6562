"""The operators at the end of a fine-tuning step, as cases that can be timed and compared: the
update of many tensors in one pass (states in 32 bits and in 8), the gradient norm with its clip
factor, token log-probabilities and the clipped policy loss with its gradient.

`own` False: elementary torch operations in 32 bits.  `own` True: the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BETA1, BETA2, EPS, LR, DECAY, STEP0 = 0.9, 0.999, 1e-8, 1e-3, 0.01, 100
MAX_NORM = 1.0
BLOCK8 = 256                      # elements that share one scale of an 8-bit state
M_TOP, V_TOP = 448.0, 1.875       # largest code value of m (e4m3) and of v (5 exponent bits, 3 mantissa bits)
F32_MAX = 3.4028234663852886e38
CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.2, 0.05
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases -------------------------------------------------------------------------------------

def listed():
    return [
        # the norm scales and biases of eight GPT-2-XL-shaped blocks: a few hundred kB, latency counts
        dict(name="step32 norms and biases", op="step32", kind="vectors", h=1600, blocks=8, grad="f32", copy=False, clip=False, packed=False),
        # one GPT-2-XL-shaped block with biases and norms, clipped, with the bf16 weights of the next forward pass
        dict(name="step32 gpt2xl block", op="step32", kind="gpt", h=1600, blocks=1, grad="bf16", copy=True, clip=True, packed=False),
        # twelve of its 48 blocks (369 M parameters, 144 tensors)
        dict(name="step32 12 gpt2xl blocks", op="step32", kind="gpt", h=1600, blocks=12, grad="bf16", copy=False, clip=True, packed=False),
        # many tensors of odd lengths from one element on (adapters, gates, embeddings of odd vocabularies)
        dict(name="step8 odd tensors", op="step8", kind="ragged", count=61, largest=60_001, pick=3, grad="f32", copy=False, clip=True, packed=False),
        # one GPT-2-XL-shaped block, 8-bit states, bf16 weight copy
        dict(name="step8 gpt2xl block", op="step8", kind="gpt", h=1600, blocks=1, grad="bf16", copy=True, clip=True, packed=False),
        # two Llama-7B-shaped blocks (405 M parameters)
        dict(name="step8 2 llama blocks", op="step8", kind="llama", h=4096, f=11008, blocks=2, grad="bf16", copy=False, clip=False, packed=False),
        # clip factor over odd fp32 gradients packed back to back (no alignment)
        dict(name="norm odd tensors", op="norm", kind="ragged", count=150, largest=40_009, pick=5, grad="f32", packed=True),
        # clip factor over twelve GPT-2-XL-shaped blocks
        dict(name="norm 12 gpt2xl blocks", op="norm", kind="gpt", h=1600, blocks=12, grad="bf16", packed=False),
        # the log-probability of a token just sampled, GPT-2's vocabulary
        dict(name="logprobs one token", op="logprobs", tokens=1, vocab=50257, logits="f32", pad=0, pitch=0, scale=1.0),
        # the old policy's pass over a batch, sampled at temperature 0.8, vocabulary padded with -inf columns
        dict(name="logprobs 4096x50304", op="logprobs", tokens=4096, vocab=50304, logits="bf16", pad=47, pitch=0, scale=1.25),
        # a few tokens with a 128 Ki vocabulary in fp32, gradient in bf16 (the dY of the weight-gradient call)
        dict(name="policy 33x131072", op="policy", tokens=33, vocab=131072, logits="f32", out="bf16", pad=0, pitch=0, scale=1.0, ref=True),
        # a training batch, GPT-2's vocabulary: odd rows, a quarter of the tokens are prompt and masked
        dict(name="policy 8192x50257", op="policy", tokens=8192, vocab=50257, logits="bf16", out="bf16", pad=0, pitch=0, scale=1.0, ref=True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["step32", "step8", "norm", "logprobs", "policy"])
    if op in ("step32", "step8", "norm"):
        kind = rng.choice(["ragged", "gpt", "llama", "vectors"])
        grad = rng.choice(["f32", "bf16"])
        case = dict(op=op, kind=kind, grad=grad, packed=op != "step8" and rng.random() < 0.3)
        if op != "norm":
            case.update(copy=rng.random() < 0.5, clip=rng.random() < 0.5)
        if kind == "ragged":
            case.update(count=_log_between(rng, 1, 300), largest=_log_between(rng, 2, 1_000_000), pick=rng.randrange(1 << 20))
        else:
            h = _log_between(rng, 40, 4096)
            h += h in (768, 1024, 3072)
            case["h"] = h
            if kind == "llama":
                case["f"] = (8 * h) // 3 + 1
            per_block = {"gpt": 12 * h * h, "llama": 12 * h * h, "vectors": 13 * h}[kind]
            case["blocks"] = _log_between(rng, 1, max(1, min(25, 300_000_000 // per_block)))
        return case
    vocab = _log_between(rng, 500, 160_000)
    vocab += vocab == 3072
    tokens = _log_between(rng, 1, max(2, min(8192, 380_000_000 // vocab)))
    tokens += tokens == 3072
    case = dict(op=op, tokens=tokens, vocab=vocab, logits=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 50]),
                pitch=rng.choice([0, 0, 1, 24]), scale=rng.choice([1.0, 1.25, 0.5]))
    if case["logits"] == "f32":
        case["tokens"] = max(1, tokens // 2)
    if op == "policy":
        case.update(out=rng.choice(["bf16", case["logits"]]), ref=rng.random() < 0.7)
    return case


def _sizes(case):
    """Lengths of the case's tensors, in the order of the list."""
    if case["kind"] == "ragged":
        r = random.Random(case["pick"])
        sizes = [_log_between(r, 1, case["largest"]) for _ in range(case["count"] - 1)] + [case["largest"]]
        return [n + (n == 3072) for n in sizes]
    h = case["h"]
    one = {"gpt": [3 * h * h, 3 * h, h * h, h, 4 * h * h, 4 * h, 4 * h * h, h, h, h, h, h],
           "llama": [h * h] * 4 + [h * case.get("f", h)] * 3 + [h, h],
           "vectors": [3 * h, h, 4 * h, h, h, h, h, h]}[case["kind"]]
    return one * case["blocks"]


def _layout(case):
    """Sizes, start of each tensor in the flat buffer that holds them all, and that buffer's length."""
    step = 1 if case["packed"] else BLOCK8
    sizes, starts, at = _sizes(case), [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // step) * step
    return sizes, starts, at


def _live(case):
    """Rows that are answers: a batch of eight sequences whose first quarter is prompt."""
    seq = max(1, case["tokens"] // 8)
    return [t for t in range(case["tokens"]) if t % seq >= seq // 4]


def work(case):
    if case["op"] in ("step32", "step8", "norm"):
        n = sum(_sizes(case))
        grad = 2 if case["grad"] == "bf16" else 4
        if case["op"] == "norm":
            return {"bytes": n * grad + 8, "flops": 2 * n}
        copy = 2 if case["copy"] else 0
        if case["op"] == "step32":
            return {"bytes": n * (grad + 24 + copy), "flops": 15 * n}
        # codes in and out, the scales, and the moments that the pass returns as the values they stand for
        return {"bytes": n * (grad + 8 + copy + 4 + 8) + 16 * sum(-(-k // BLOCK8) for k in _sizes(case)), "flops": 30 * n}
    esize = 2 if case["logits"] == "bf16" else 4
    if case["op"] == "logprobs":
        return {"bytes": case["tokens"] * (case["vocab"] * esize + 20), "flops": 6 * case["tokens"] * case["vocab"]}
    osize = 2 if case["out"] == "bf16" else 4
    live = len(_live(case))
    return {"bytes": live * case["vocab"] * esize + case["tokens"] * (case["vocab"] * osize + 32),
            "flops": 9 * live * case["vocab"]}


# ---- inputs ------------------------------------------------------------------------------------

def _encode_v(v, top):
    """Nearest code of v*(1.875/top): 5 exponent bits, 3 mantissa bits, ties to even; 0 only for 0."""
    y = v * (torch.reciprocal(top) * V_TOP).clamp(max=F32_MAX)
    bits = y.view(torch.int32)
    code = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - (96 << 3)
    return torch.where(v > 0, code.clamp(1, 255), 0).to(torch.uint8)


def _encode_m(m, top):
    return (m * (torch.reciprocal(top) * M_TOP).clamp(max=F32_MAX)).to(torch.float8_e4m3fn)


def _decode_v(code):
    bits = (code.to(torch.int32) << 20) + (96 << 23)
    return torch.where(code > 0, bits.view(torch.float32), 0.0)


def _lists(s, names):
    return [[s[k][o:o + n] for o, n in zip(s["starts"], s["sizes"])] for k in names]


def _prepare_step(case, gen):
    sizes, starts, total = _layout(case)
    s = {"case": case, "sizes": sizes, "starts": starts, "t": STEP0}
    grid = torch.zeros(total, dtype=torch.int32, device="cuda")  # 1 where a tensor begins: how large its gradients are
    inside = torch.zeros(total + 1, dtype=torch.int32, device="cuda")
    at = torch.tensor(starts, device="cuda")
    end = at + torch.tensor(sizes, device="cuda")
    one = torch.ones(len(sizes), dtype=torch.int32, device="cuda")
    grid.index_add_(0, at, one)
    inside.index_add_(0, at, one).index_add_(0, end, -one)
    inside = inside.cumsum(0)[:total] > 0
    spread = torch.exp(torch.randn(len(sizes), device="cuda", generator=gen))
    size = 1e-3 * spread[(grid.cumsum(0) - 1)] * inside
    del grid, inside

    def normal():
        return torch.randn(total, device="cuda", generator=gen)

    g = normal().mul_(size)
    g[::97] = 0.0                                   # entries that this batch does not reach
    s["g"] = g.to(DTYPES[case["grad"]])
    del g
    if case["op"] == "norm":
        return s
    s["w"] = normal().mul_(0.02).mul_(size > 0)
    m = normal().mul_(size).mul_(0.3)
    v = normal().mul_(size).square_().add_(0.1 * size * size)
    s["factor"] = torch.full((1,), 0.37, device="cuda") if case["clip"] else None
    if case["op"] == "step32":
        s["m"], s["v"] = m, v
    else:
        m, v = m.view(-1, BLOCK8), v.view(-1, BLOCK8)
        mt, vt = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
        s["m8"], s["v8"] = _encode_m(m, mt).view(-1), _encode_v(v, vt).view(-1)
        s["ms"], s["vs"] = (mt * (1 / M_TOP)).view(-1), (vt * (1 / V_TOP)).view(-1)
    s["wb"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda") if case["copy"] else None
    return s


def _prepare_rows(case, gen):
    T, V = case["tokens"], case["vocab"]
    rows = torch.randn(T, V + case["pitch"], device="cuda", generator=gen, dtype=DTYPES[case["logits"]]).mul_(2)
    logits = rows[:, :V]
    real = V - case["pad"]
    targets = torch.randint(0, real, (T,), device="cuda", generator=gen)
    at = torch.arange(T, device="cuda")
    logits[at, targets] += 8 * torch.rand(T, device="cuda", generator=gen).to(logits.dtype)
    if case["pad"]:
        logits[:, real:] = -math.inf                 # columns that only pad the vocabulary
    s = {"case": case, "logits": logits, "targets": targets}
    if case["op"] == "logprobs":
        s["logp"], s["lse"], s["entropy"] = (torch.empty(T, device="cuda") for _ in range(3))
        return s
    logp = torch.cat([_row_logp(x, t, case["scale"]) for x, t in zip(logits.split(1024), targets.split(1024))])

    def drift(size, shift):
        # on a grid of 1/512 whose points lie off log(1-0.2) and log(1+0.2): every form takes the same branch
        return (torch.round(torch.randn(T, device="cuda", generator=gen) * (512 * size)) + shift) / 512

    s["old"] = logp - drift(0.15, 0.5)
    s["ref"] = logp - drift(0.3, 0.5) if case["ref"] else None
    s["adv"] = torch.randn(T, device="cuda", generator=gen) + 0.2
    live = torch.tensor(_live(case), device="cuda")
    s["weights"] = torch.zeros(T, device="cuda").index_fill_(0, live, 1.0 / live.numel())
    s["dlogits"] = torch.empty(T, V, dtype=DTYPES[case["out"]], device="cuda")
    s["stats"], s["logp"] = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    return s


def _row_logp(x, t, scale):
    z = x.float() * scale
    return z.gather(1, t[:, None])[:, 0] - torch.logsumexp(z, 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) & 0x7FFFFFFF)
    s = (_prepare_rows if case["op"] in ("logprobs", "policy") else _prepare_step)(case, gen)
    if own:  # the context and the marshalled lists, which a training program makes once
        import paper_2305_19982_b200 as adama
        s["opt"] = adama.AdamA(BETA1, BETA2, EPS)
        s["opt"].set_weight_decay(DECAY)
        s["opt"].set_step(STEP0)
        if "sizes" in s:
            s["G"] = adama.TensorList(_lists(s, "g")[0])
        if case["op"] == "norm":
            s["out"] = torch.empty(4, device="cuda")
        if case["op"] in ("step32", "step8"):
            s["W"] = adama.TensorList(_lists(s, "w")[0])
            s["WB"] = adama.TensorList(_lists(s, ["wb"])[0]) if case["copy"] else None
        if case["op"] == "step32":
            s["M"], s["V"] = (adama.TensorList(x) for x in _lists(s, ["m", "v"]))
        if case["op"] == "step8":
            scales = [[s[k][o // BLOCK8:o // BLOCK8 + -(-n // BLOCK8)] for o, n in zip(s["starts"], s["sizes"])] for k in ("ms", "vs")]
            s["S"] = adama.State8List([adama.State8(*x) for x in zip(*_lists(s, ["m8"]), scales[0], *_lists(s, ["v8"]), scales[1])])
            s["m"], s["v"] = torch.zeros_like(s["w"]), torch.zeros_like(s["w"])
            s["M"], s["V"] = (adama.TensorList(x) for x in _lists(s, ["m", "v"]))
    return s


# ---- the library's calls -----------------------------------------------------------------------

def _own_step32(s):
    s["opt"].begin_minibatch(1)
    s["opt"].fold_apply_multi(s["W"], s["G"], s["M"], s["V"], LR, w_bf16=s["WB"], grad_factor=s["factor"])
    return {"w": s["w"], "m": s["m"], "v": s["v"], "copy": s["wb"]}


def _own_step8(s):
    s["opt"].begin_minibatch(1)
    s["opt"].fold_apply8_multi(s["W"], s["G"], s["S"], LR, w_bf16=s["WB"], grad_factor=s["factor"])
    s["opt"].state8_unpack_multi(s["S"], s["M"], s["V"])
    return {"w": s["w"], "m": s["m"], "v": s["v"], "copy": s["wb"]}


def _own_norm(s):
    s["opt"].grad_norm_multi(s["G"], MAX_NORM, s["out"])
    return s["out"][:2]


def _own_logprobs(s):
    s["opt"].token_logprobs(s["logits"], s["targets"], s["logp"], lse=s["lse"], entropy=s["entropy"], logit_scale=s["case"]["scale"])
    return {"logp": s["logp"], "lse": s["lse"], "entropy": s["entropy"]}


def _own_policy(s):
    s["opt"].policy_loss(s["logits"], s["targets"], s["old"], s["adv"], s["weights"], s["dlogits"], s["stats"],
                         ref_logp=s["ref"], logp=s["logp"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL_COEF,
                         logit_scale=s["case"]["scale"])
    return {"dlogits": s["dlogits"], "stats": s["stats"], "logp": s["logp"]}


# ---- the plain forms: elementary operations in 32 bits -------------------------------------------

def _constants(t):
    return {"a": 1 - BETA1, "b": 1 - BETA2, "step": LR / (1 - BETA1 ** t), "ibc2": 1 / (1 - BETA2 ** t), "keep": 1 - LR * DECAY}


def _plain_update(s, m, v):
    """Adds the gradient to m and v, updates s["w"]; returns the new m and v before their decay."""
    s["t"] += 1
    c = _constants(s["t"])
    g = s["g"].float().view(m.shape)
    if s["factor"] is not None:
        g = g * s["factor"]
    m = m + g * c["a"]
    v = v + (g * c["b"]) * g
    w = s["w"].view(m.shape) * c["keep"] - m / (torch.sqrt(v * c["ibc2"]) + EPS) * c["step"]
    s["w"] = w.view(-1)
    return m, v


def _plain_step32(s):
    m, v = _plain_update(s, s["m"], s["v"])
    s["m"], s["v"] = m * BETA1, v * BETA2
    return {"w": s["w"], "m": s["m"], "v": s["v"], "copy": s["w"].bfloat16() if s["case"]["copy"] else None}


def _plain_step8(s):
    m = s["m8"].float().view(-1, BLOCK8) * s["ms"][:, None]
    v = _decode_v(s["v8"]).view(-1, BLOCK8) * s["vs"][:, None]
    m, v = _plain_update(s, m, v)
    mt, vt = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
    s["m8"], s["v8"] = _encode_m(m, mt).view(-1), _encode_v(v, vt).view(-1)
    s["ms"], s["vs"] = (mt * (1 / M_TOP) * BETA1).view(-1), (vt * (1 / V_TOP) * BETA2).view(-1)
    m = s["m8"].float().view(-1, BLOCK8) * s["ms"][:, None]
    v = _decode_v(s["v8"]).view(-1, BLOCK8) * s["vs"][:, None]
    return {"w": s["w"], "m": m.view(-1), "v": v.view(-1), "copy": s["w"].bfloat16() if s["case"]["copy"] else None}


def _plain_norm(s):
    norm = s["g"].float().square().sum().sqrt()
    return torch.stack([norm, torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)])


def _softmax_parts(x, scale):
    """z - max, exp(z - max), the sum of those, for z = scale * x."""
    z = x.float() * scale
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    return z, top[:, 0], e, e.sum(1)


def _plain_logprobs(s):
    z, top, e, total = _softmax_parts(s["logits"], s["case"]["scale"])
    lse = top + torch.log(total)
    logp = z.gather(1, s["targets"][:, None])[:, 0] - lse
    entropy = lse - torch.where(e > 0, e * z, 0.0).sum(1) / total
    return {"logp": logp, "lse": lse, "entropy": entropy}


def _plain_policy(s):
    scale, wt, adv = s["case"]["scale"], s["weights"], s["adv"]
    live = wt != 0
    z, top, e, total = _softmax_parts(s["logits"], scale)
    logp = z.gather(1, s["targets"][:, None])[:, 0] - top - torch.log(total)
    ratio = torch.exp(logp - s["old"])
    clipped = ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
    cut = ratio * adv > clipped
    pg = -torch.minimum(ratio * adv, clipped)
    slope = torch.where(cut, 0.0, -ratio * adv)
    kl = torch.zeros_like(pg)
    if s["ref"] is not None:
        d = s["ref"] - logp
        kl = torch.exp(d) - d - 1
        slope = slope + KL_COEF * (1 - torch.exp(d))
    row = torch.where(live, wt * slope * scale, 0.0)
    grad = e * (-row / total)[:, None]
    grad.scatter_add_(1, s["targets"][:, None], row[:, None])
    terms = torch.stack([pg + KL_COEF * kl, pg, kl, cut.float()])
    stats = torch.where(live, terms * wt, 0.0).sum(1)
    return {"dlogits": grad.to(DTYPES[s["case"]["out"]]), "stats": stats, "logp": torch.where(live, logp, 0.0)}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"step32": _own_step32, "step8": _own_step8, "norm": _own_norm, "logprobs": _own_logprobs, "policy": _own_policy}[op](s)
    return {"step32": _plain_step32, "step8": _plain_step8, "norm": _plain_norm, "logprobs": _plain_logprobs, "policy": _plain_policy}[op](s)


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _nearest(x, values):
    """The value nearest to x in an ascending table; the larger of two equally near."""
    middle = (values[1:] + values[:-1]) / 2
    return values[torch.bucketize(x, middle, right=True)]


def _exact_step(s, case):
    # the hyper-parameters' derived constants are 32-bit numbers by definition of the call
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    t = STEP0 + 1
    g = s["g"].double() * (float(s["factor"]) if case["clip"] else 1.0)
    if case["op"] == "step32":
        m, v = s["m"].double(), s["v"].double()
    else:
        kinds = torch.arange(256, device="cuda")
        v_values = torch.where(kinds > 0, (1 + (kinds % 8).double() / 8) * torch.exp2((kinds // 8 - 31).double()), 0.0)
        m = s["m8"].double() * s["ms"].double().repeat_interleave(BLOCK8)
        v = v_values[s["v8"].long()] * s["vs"].double().repeat_interleave(BLOCK8)
    m += f32(1 - BETA1) * g
    v += f32(1 - BETA2) * g * g
    del g
    w = s["w"].double() * f32(1 - LR * DECAY)
    w -= f32(LR / (1 - BETA1 ** t)) * m / ((v * f32(1 / (1 - BETA2 ** t))).sqrt() + f32(EPS))
    if case["op"] == "step8":
        e4m3 = torch.arange(127, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).double()
        e4m3 = torch.cat([-e4m3[1:].flip(0), e4m3])
        m, v = m.view(-1, BLOCK8), v.view(-1, BLOCK8)
        sm, sv = m.abs().amax(1, keepdim=True) / M_TOP, v.amax(1, keepdim=True) / V_TOP
        safe = lambda x: torch.where(x > 0, x, 1.0)  # noqa: E731
        m = (_nearest(m / safe(sm), e4m3) * sm).view(-1)
        low = _nearest(v / safe(sv), v_values).clamp(min=float(v_values[1]))
        v = torch.where(v > 0, low * sv, 0.0).view(-1)
    return {"w": w, "m": m * BETA1, "v": v * BETA2, "copy": w if case["copy"] else None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("step32", "step8"):
        return _exact_step(s, case)
    if case["op"] == "norm":
        norm = s["g"].double().norm()
        return torch.stack([norm, torch.clamp(MAX_NORM / norm, max=1.0)])
    scale, at, parts = case["scale"], 0, []
    for x in s["logits"].split(max(1, 40_000_000 // case["vocab"])):
        rows = slice(at, at + x.shape[0])
        at += x.shape[0]
        z = x.double() * scale
        lse = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[:, None])
        logp = z.gather(1, s["targets"][rows, None])[:, 0] - lse
        if case["op"] == "logprobs":
            parts.append((logp, lse, -torch.xlogy(p, p).sum(1)))
            continue
        old, adv, wt = (s[k][rows].double() for k in ("old", "adv", "weights"))
        ratio = (logp - old).exp()
        inside = (adv >= 0) & (ratio <= 1 + CLIP_HIGH) | (adv < 0) & (ratio >= 1 - CLIP_LOW)
        limit = torch.where(adv >= 0, 1 + CLIP_HIGH, 1 - CLIP_LOW)
        pg = -adv * torch.where(inside, ratio, limit)
        slope, kl = -adv * ratio * inside, torch.zeros_like(pg)
        if s["ref"] is not None:
            d = s["ref"][rows].double() - logp
            kl = torch.expm1(d) - d
            slope = slope - KL_COEF * torch.expm1(d)
        p.neg_().scatter_add_(1, s["targets"][rows, None], torch.ones_like(logp)[:, None])
        p.mul_((wt * slope * scale)[:, None])
        stats = (torch.stack([pg + KL_COEF * kl, pg, kl, (~inside).double()]) * wt).sum(1)
        parts.append((p, stats, torch.where(wt != 0, logp, 0.0)))
    if case["op"] == "logprobs":
        return dict(zip(("logp", "lse", "entropy"), (torch.cat(x) for x in zip(*parts))))
    return {"dlogits": torch.cat([x[0] for x in parts]), "stats": sum(x[1] for x in parts), "logp": torch.cat([x[2] for x in parts])}
