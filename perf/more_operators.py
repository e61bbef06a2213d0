"""What a compressed language model is judged by and tuned with, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` names what the user's program calls:

  score           log probabilities of given tokens, entropy and top alternatives of rows of logits: the judgement of a
                  compressed model's answers, and the dense model's side of a distillation
  layernorm       residual addition and layer norm, output in the inputs' type or in 8 bits for the 4-bit products
  layernorm_grad  its backward pass: gradients of the inputs, the gain and the bias
  embed           rows of an embedding table for token ids, times a scale
  embed_grad      the table's gradient: for every row of it the sum over the tokens that read it
  adamw           an AdamW step over many tensors at once, moments in 32 bits or in 8 with a scale per 256 values

`type` is that of activations, gradients and logits (adamw: of parameters and gradients); statistics, gains, biases and
32-bit moments are fp32.  Ids are int32; a negative one is no token.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256      # values that share a scale, of moments in 8 bits
TOP8 = 448.0     # the largest number of the 8-bit type


def listed():
    return [
        # one generated token's log probability and alternatives: latency is all it costs
        {"name": "score_1x32000_f32", "kind": "score", "tokens": 1, "vocab": 32000, "top": 20, "type": "f32",
         "temperature": 1.0},
        # the dense model's top logits for a training batch, as the distillation takes them
        {"name": "score_2048x131072_bf16", "kind": "score", "tokens": 2048, "vocab": 131072, "top": 64, "type": "bf16",
         "temperature": 2.0},
        # one token through a BERT-base sized transformer's norm
        {"name": "layernorm_1x768_f16", "kind": "layernorm", "tokens": 1, "cols": 768, "type": "f16", "bits8": False},
        # a training batch's norm with its residual stream
        {"name": "layernorm_4096x8192_bf16", "kind": "layernorm", "tokens": 4096, "cols": 8192, "type": "bf16",
         "bits8": False},
        # the backward pass of a small ragged batch
        {"name": "layernorm_grad_333x1283_f32", "kind": "layernorm_grad", "tokens": 333, "cols": 1283, "type": "f32"},
        # and of a training batch
        {"name": "layernorm_grad_4096x4096_bf16", "kind": "layernorm_grad", "tokens": 4096, "cols": 4096, "type": "bf16"},
        # a decoding step of eight sequences, rows not aligned to anything
        {"name": "embed_8x1283_bf16", "kind": "embed", "tokens": 8, "vocab": 32000, "cols": 1283, "type": "bf16"},
        # a training batch from a large table
        {"name": "embed_16384x4096_bf16", "kind": "embed", "tokens": 16384, "vocab": 131072, "cols": 4096,
         "type": "bf16"},
        # a short sequence's gradient into a small table
        {"name": "embed_grad_100x768_f32", "kind": "embed_grad", "tokens": 100, "vocab": 5000, "cols": 768, "type": "f32",
         "out": "f32"},
        # a training batch's, sums kept in 32 bits
        {"name": "embed_grad_16384x4096_bf16", "kind": "embed_grad", "tokens": 16384, "vocab": 32000, "cols": 4096,
         "type": "bf16", "out": "f32"},
        # gains and biases of the norms of a small transformer
        {"name": "adamw_50x768_f32", "kind": "adamw", "tensors": 50, "size": 768, "type": "f32", "bits": 32,
         "master": False},
        # an embedding table in half the bits with fp32 copies, moments in 8
        {"name": "adamw_4x16000000_bf16", "kind": "adamw", "tensors": 4, "size": 16000000, "type": "bf16", "bits": 8,
         "master": True},
    ]


# bounds on what draw() may give: half of the largest listed sets of logits, activations, tables and parameters
_MOST_LOGITS = 2 ** 27
_MOST_ACTIVATIONS = 2 ** 24
_MOST_TABLE = 2 ** 27
_MOST_PARAMETERS = 2 ** 25


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["score", "score", "layernorm", "layernorm_grad", "embed", "embed_grad", "embed_grad", "adamw", "adamw"])
    case = {"kind": kind, "type": rng.choice(["bf16", "f16", "f32"])}
    if kind == "score":
        case["vocab"] = _log_int(rng, 1000, 131072)
        case["tokens"] = _log_int(rng, 1, min(4096, _MOST_LOGITS // case["vocab"]))
        case["top"] = _log_int(rng, 1, 256)
        case["temperature"] = round(rng.uniform(0.5, 4.0), 2)
    elif kind in ("layernorm", "layernorm_grad"):
        case["cols"] = _log_int(rng, 64, 16384)
        case["tokens"] = _log_int(rng, 1, min(8192, _MOST_ACTIVATIONS // case["cols"]))
        if kind == "layernorm":
            case["bits8"] = case["type"] != "f32" and rng.random() < 0.5
    elif kind in ("embed", "embed_grad"):
        case["cols"] = _log_int(rng, 64, 8192)
        case["vocab"] = _log_int(rng, 1000, min(262144, _MOST_TABLE // case["cols"]))
        case["tokens"] = _log_int(rng, 1, min(32768, 2 * _MOST_ACTIVATIONS // case["cols"]))
        if kind == "embed_grad":
            case["out"] = rng.choice(["f32", case["type"]])
    else:
        case["size"] = _log_int(rng, 64, 2 ** 23)
        case["tensors"] = _log_int(rng, 1, min(200, _MOST_PARAMETERS // case["size"]))
        case["bits"] = rng.choice([8, 32])
        case["master"] = case["type"] != "f32" and rng.random() < 0.6
    return case


# ------------------------------------------------------------------------------------------- inputs
def _tokens(T, d, gen):
    """Activations of a transformer: a few channels are ten times the others, and all lie a little off zero."""
    x = torch.randn(T, d, generator=gen, device=DEV).add_(0.2)
    heavy = torch.randperm(d, generator=gen, device=DEV)[:max(1, round(0.01 * d))]
    x[:, heavy] *= 10.0
    return x


def _ids(T, V, gen):
    """Tokens of a text: an id's share falls with its rank; a sixteenth of the places hold no token."""
    u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)
    ids = torch.exp(u * math.log(V + 1.0)).floor_().sub_(1.0).clamp_(0, V - 1).to(torch.int32)
    return torch.where(torch.rand(T, generator=gen, device=DEV) < 0.0625, -1, ids)


def sizes_of(case):
    """Values of each tensor: all of the case's size, or an eighth to three less, odd numbers among them."""
    n = case["size"]
    return [n - (i % 4) * (n // 8) - i % 2 for i in range(case["tensors"])]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kind, dt = case["kind"], TYPES[case["type"]]
    s = {"case": case}
    if own:
        import paper_2208_11580_amd as obc
        s["ctx"] = obc.Context()
    if kind == "adamw":
        return _prepare_adamw(case, gen, s)
    T = case["tokens"]
    if kind == "score":
        V = case["vocab"]
        z = torch.randn(T, V, generator=gen, device=DEV).mul_(3.0)
        # the vocabulary is padded to a round number: what lies behind the last token is masked
        z[:, V - V // 200:] = float("-inf")
        s["z"] = z.to(dt)
        # a batch's tokens are likely ones, an eighth of them belong to the prompt and do not count
        drawn = (z.mul_(0.7) - torch.rand(T, V, generator=gen, device=DEV).clamp_min_(1e-9).log_().neg_().log_()).argmax(1)
        s["target"] = torch.where(torch.rand(T, generator=gen, device=DEV) < 0.125, -1, drawn).to(torch.int32)
        if own:
            k = case["top"]
            s["out"] = {"logp": torch.empty(T, device=DEV), "entropy": torch.empty(T, device=DEV), "lse": torch.empty(T, device=DEV),
                        "top_index": torch.empty(T, k, dtype=torch.int32, device=DEV), "top_logit": torch.empty(T, k, device=DEV)}
        return s
    d = case["cols"]
    if kind in ("embed", "embed_grad"):
        V = case["vocab"]
        s["ids"] = _ids(T, V, gen)
        s["scale"] = float(d) ** 0.5
        if kind == "embed":
            s["table"] = torch.randn(V, d, generator=gen, device=DEV).mul_(d ** -0.5).to(dt)
            if own:
                s["out"] = torch.empty(T, d, dtype=dt, device=DEV)
        else:
            s["dy"] = (torch.randn(T, d, generator=gen, device=DEV) * 1e-3).to(dt)
            if own:
                s["out"] = torch.empty(V, d, dtype=TYPES[case["out"]], device=DEV)
        return s
    s["gain"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device=DEV)
    if kind == "layernorm_grad":
        h = _tokens(T, d, gen).to(dt)
        f = h.double()
        mean = f.mean(1)
        s["h"], s["mean"] = h, mean.float()
        s["rstd"] = ((f - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
        s["dy"] = (torch.randn(T, d, generator=gen, device=DEV) * 1e-3).to(dt)
        s["dh"] = (torch.randn(T, d, generator=gen, device=DEV) * 1e-3).to(dt)
        if own:
            s["out"] = {"dx": torch.empty(T, d, dtype=dt, device=DEV), "dgain": torch.empty(d, device=DEV),
                        "dbias": torch.empty(d, device=DEV)}
        return s
    s["bias"] = 0.1 * torch.randn(d, generator=gen, device=DEV)
    s["x"] = _tokens(T, d, gen).mul_(0.3).to(dt)
    s["residual"] = _tokens(T, d, gen).to(dt)
    if own:
        s["out"] = {"h": torch.empty(T, d, dtype=dt, device=DEV),
                    "y": torch.empty(T, d, dtype=torch.int8 if case["bits8"] else dt, device=DEV)}
        if case["bits8"]:
            s["out"]["scale"] = torch.empty(T, device=DEV)
    return s


def _prepare_adamw(case, gen, s):
    dt, F8 = TYPES[case["type"]], torch.float8_e4m3fn
    s["step"], s["seed"] = 1000, 7
    s["grad_scale"] = torch.full((1,), 0.37, device=DEV)
    for name in ("p", "master", "g", "m", "v", "m_scale", "v_scale"):
        s[name] = []
    for n in sizes_of(case):
        p = torch.randn(n, generator=gen, device=DEV).mul_(0.03)
        s["p"].append(p.to(dt))
        s["master"].append(p if case["master"] else None)
        s["g"].append(torch.randn(n, generator=gen, device=DEV).mul_(1e-3).to(dt))
        # magnitudes of gradients differ from weight to weight by orders
        r = torch.randn(n, generator=gen, device=DEV).mul_(1.5).exp_().mul_(3e-4)
        m = torch.randn(n, generator=gen, device=DEV).mul_(r).mul_(0.3)
        if case["bits"] == 32:
            s["m"].append(m)
            s["v"].append(r.square_())
            continue
        blocks = -(-n // BLOCK)
        for name, x in (("m", m), ("v", r)):
            pad = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).view(blocks, BLOCK)
            scale = pad.abs().amax(1) / TOP8
            s[name].append((pad / scale[:, None]).clamp_(-TOP8, TOP8).view(-1)[:n].to(F8))
            s[name + "_scale"].append(scale)
    if own:
        import paper_2208_11580_amd as obc
        at = lambda name, i: s[name][i] if s[name] else None  # noqa: E731
        s["states"] = [obc.AdamState(s["m"][i], s["v"][i], at("m_scale", i), at("v_scale", i), s["master"][i])
                       for i in range(case["tensors"])]
        # out of place, as a program does that keeps the last step's weights to go back to
        s["plan"] = s["ctx"].obc_adamw_plan(s["p"], s["g"], s["states"], decay=DECAY, out=(
            [torch.empty_like(p) for p in s["p"]],
            [obc.AdamState(*[None if t is None else torch.empty_like(t) for t in st]) for st in s["states"]]))
    return s


# --------------------------------------------------------------------------------- the framework's kernels
def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    kind = case["kind"]
    if kind == "score":
        return ctx.obc_score(s["z"], s["target"], top=case["top"], temperature=case["temperature"], out=s["out"])
    if kind == "embed":
        return ctx.obc_embed(s["table"], s["ids"], scale=s["scale"], out=s["out"])
    if kind == "embed_grad":
        return ctx.obc_embed_grad(s["ids"], s["dy"], case["vocab"], scale=s["scale"], out=s["out"])
    if kind == "layernorm_grad":
        return ctx.obc_layernorm_grad(s["h"], s["gain"], s["mean"], s["rstd"], s["dy"], dh=s["dh"], out=s["out"])
    if kind == "layernorm":
        r = ctx.obc_layernorm(s["x"], s["gain"], s["bias"], eps=EPS, residual=s["residual"], quant8=case["bits8"], out=s["out"])
        # (8 bits: the values that they stand for)
        return {"h": r["h"], "y": (r["y"] * r["scale"][:, None]).to(r["h"].dtype) if case["bits8"] else r["y"]}
    p, states = ctx.obc_adamw(s["plan"], s["step"], LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, grad_scale=s["grad_scale"],
                              seed=s["seed"])
    return _adamw_outputs(p, [st.m for st in states], [st.v for st in states], [st.m_scale for st in states],
                          [st.v_scale for st in states], [st.master for st in states])


def _adamw_outputs(p, m, v, m_scale, v_scale, master):
    """The largest and the smallest tensor's results, and all parameters."""
    r = {"p": p[:40], "m": m[0], "v": v[0], "m_last": m[-1], "v_last": v[-1], "master": master[:10]}
    if m_scale[0] is not None:
        r.update(m_scale=m_scale[0], v_scale=v_scale[0])
    return r


# ------------------------------------------------------------------------------------------ the plain forms
def _score(s):
    case, tau, k = s["case"], s["case"]["temperature"], s["case"]["top"]
    T, V = s["z"].shape
    z = s["z"].float() + 0.0      # (one zero only)
    # larger logits first, lower indices first among equal ones: both in one whole number
    bits = z.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 32) + torch.arange(V - 1, -1, -1, device=DEV)
    top = V - 1 - (key.topk(min(k, V), dim=1).values & 0xffffffff)
    del key, bits
    top = torch.nn.functional.pad(top, (0, k - top.shape[1]))
    top_logit = torch.gather(z, 1, top)
    top_index = torch.where((top_logit == float("-inf")) | (torch.arange(k, device=DEV) >= V), -1, top).to(torch.int32)
    z /= tau
    d = z - z.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1)
    lse = z.amax(1) + total.log()
    entropy = total.log() - (e * d.clamp_min(-1e30)).sum(1) / total
    target = s["target"]
    logp = torch.gather(d, 1, target.clamp_min(0).long()[:, None])[:, 0] - total.log()
    return {"logp": torch.where(target >= 0, logp, 0.0), "entropy": entropy, "lse": lse, "top_index": top_index,
            "top_logit": top_logit}


def _round8(y):
    """The values of y rounded to 8 bits with a scale for each row."""
    top = y.abs().amax(1, keepdim=True)
    scale = torch.where(top > 0, top / 127.0, 1.0)
    return torch.round(y / scale).clamp(-127, 127) * scale


# odd parts of the fractions of the golden ratio, of the roots of 2, 3 and 5, and of pi
_MIX = (0x9E3779B1, 0x6A09E667, 0xBB67AE85, 0x3C6EF373, 0x243F6A89)


def dither(n, seed, step, ordinal):
    """32 bits for each of a tensor's n values: the lower 16 dither the first moment, the upper 16 the second."""
    low = 0xffffffff
    key = (seed * _MIX[1] + step * _MIX[2] + ordinal * _MIX[3]) & low
    h = torch.arange(n, device=DEV) ^ key
    h = (h * _MIX[0]) & low
    h ^= h >> 15
    h = (h * _MIX[1]) & low
    h ^= h >> 14
    h = (h * _MIX[4]) & low
    h ^= h >> 16
    return h


def _round_moment(x, u, floor):
    """x on the 8-bit type's grid times a scale per block, up or down by the dither u (0 .. 65535); floor: what is not
    zero does not become zero."""
    n = x.numel()
    blocks = -(-n // BLOCK)
    pad = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).view(blocks, BLOCK)
    scale = pad.abs().amax(1) / TOP8
    a = (pad.abs() * torch.where(scale > 0, 1.0 / scale, 0.0)[:, None]).clamp_max_(TOP8).view(-1)[:n]
    # the grid's step: 8 to an octave, down to 2^-9
    q = torch.exp2(torch.frexp(a).exponent.sub_(1).clamp_min_(-6).sub_(3).float())
    y = torch.floor(a / q + u.float() / 65536.0) * q
    if floor:
        y = torch.where((a > 0) & (y == 0), 2.0 ** -9, y)
    return torch.copysign(y, x).to(torch.float8_e4m3fn), scale


def _decode(q, scale):
    return q.float() * scale.repeat_interleave(BLOCK)[:q.numel()]


def _adamw_one(s, i):
    case, t = s["case"], s["step"]
    p = s["p"][i].float() if s["master"][i] is None else s["master"][i]
    g = s["g"][i].float() * s["grad_scale"]
    bits8 = case["bits"] == 8
    m = _decode(s["m"][i], s["m_scale"][i]) if bits8 else s["m"][i]
    v = _decode(s["v"][i], s["v_scale"][i]).square() if bits8 else s["v"][i]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    c1, c2 = 1.0 / (1.0 - BETA1 ** t), (1.0 - BETA2 ** t) ** -0.5
    p = p * (1.0 - LR * DECAY) - (LR * c1) * m / (v.sqrt() * c2 + ADAM_EPS)
    out = p.to(s["p"][i].dtype), m, v, None, None, None if s["master"][i] is None else p
    if not bits8:
        return out
    u = dither(p.numel(), s["seed"], t, i)
    m8, m_scale = _round_moment(m, u & 0xffff, False)
    v8, v_scale = _round_moment(v.sqrt(), u >> 16, True)
    return out[0], m8, v8, m_scale, v_scale, out[5]


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    kind, dt = case["kind"], TYPES[case["type"]]
    if kind == "score":
        return _score(s)
    if kind == "embed":
        y = s["table"][s["ids"].clamp_min(0).long()].float() * s["scale"]
        return (y * (s["ids"] >= 0)[:, None]).to(dt)
    if kind == "embed_grad":
        total = torch.zeros(case["vocab"], case["cols"], device=DEV)
        total.index_add_(0, s["ids"].clamp_min(0).long(), s["dy"].float() * (s["ids"] >= 0)[:, None])
        return (total * s["scale"]).to(TYPES[case["out"]])
    if kind == "layernorm_grad":
        xhat = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].float()
        gy = dy * s["gain"]
        dx = gy - gy.mean(1, keepdim=True) - xhat * (gy * xhat).mean(1, keepdim=True)
        dx = s["dh"].float() + s["rstd"][:, None] * dx
        return {"dx": dx.to(dt), "dgain": (dy * xhat).sum(0), "dbias": dy.sum(0)}
    if kind == "layernorm":
        h = s["x"].float() + s["residual"].float()
        c = h - h.mean(1, keepdim=True)
        y = c * (c.square().mean(1, keepdim=True) + EPS).rsqrt() * s["gain"] + s["bias"]
        return {"h": h.to(dt), "y": (_round8(y) if case["bits8"] else y).to(dt)}
    return _adamw_outputs(*zip(*[_adamw_one(s, i) for i in range(case["tensors"])]))


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_score(case, s):
    tau, k, T = case["temperature"], case["top"], case["tokens"]
    logp, entropy, lse = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(3))
    index = torch.full((T, k), -1, dtype=torch.int32, device=DEV)
    logit = torch.full((T, k), float("-inf"), dtype=torch.float64, device=DEV)
    for a in range(0, T, 128):
        z = s["z"][a:a + 128].double()
        best, order = torch.sort(z, dim=1, descending=True, stable=True)
        n = min(k, z.shape[1])
        logit[a:a + 128, :n] = best[:, :n]
        index[a:a + 128, :n] = torch.where(best[:, :n] == float("-inf"), -1, order[:, :n]).to(torch.int32)
        z /= tau
        lse[a:a + 128] = torch.logsumexp(z, dim=1)
        lp = z - lse[a:a + 128, None]
        entropy[a:a + 128] = -torch.where(lp == float("-inf"), 0.0, lp.exp() * lp).sum(1)
        t = s["target"][a:a + 128].long()
        logp[a:a + 128] = lp.gather(1, (t * (t >= 0))[:, None])[:, 0] * (t >= 0)
    return {"logp": logp, "entropy": entropy, "lse": lse, "top_index": index, "top_logit": logit}


def _exact_adamw(case, s):
    t, outs = s["step"], []
    for i in range(case["tensors"]):
        p = (s["p"][i] if s["master"][i] is None else s["master"][i]).double()
        g = s["g"][i].double() * s["grad_scale"].double()
        n = p.numel()
        m, v = s["m"][i].double(), s["v"][i].double()
        if case["bits"] == 8:
            at = torch.arange(n, device=DEV) // BLOCK
            m = m * s["m_scale"][i].double()[at]
            v = (v * s["v_scale"][i].double()[at]) ** 2
        m = m + (g - m) * (1 - BETA1)
        v = v + (g * g - v) * (1 - BETA2)
        step = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
        p = p - LR * DECAY * p - LR * step
        scales = [None, None]
        if case["bits"] == 8:
            u = dither(n, s["seed"], t, i)
            coded = []
            for j, (x, r) in enumerate(((m, u % 65536), (v.sqrt(), u // 65536))):
                top = torch.zeros(-(-n // BLOCK), dtype=torch.float64, device=DEV)
                top.scatter_reduce_(0, at, x.abs(), "amax")
                scales[j] = top / TOP8
                a = x.abs() / scales[j][at].clamp_min(1e-300)
                q = 2.0 ** (torch.log2(a.clamp_min(2.0 ** -6)).floor() - 3)
                y = ((a / q) + r.double() / 65536).floor() * q
                if j:
                    y = torch.where(a > 0, y.clamp_min(2.0 ** -9), y)
                coded.append(torch.where(x < 0, -y, y))
            m, v = coded
        outs.append((p, m, v, scales[0], scales[1], None if s["master"][i] is None else p))
    return _adamw_outputs(*zip(*outs))


def exact(case, seed):
    global own
    kind = case["kind"]
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if kind == "score":
        return _exact_score(case, s)
    if kind == "adamw":
        return _exact_adamw(case, s)
    if kind == "embed":
        out = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device=DEV)
        real = (s["ids"] >= 0).nonzero()[:, 0]
        out[real] = s["table"].index_select(0, s["ids"][real]).double() * s["scale"]
        return out
    if kind == "embed_grad":
        # tokens in the order of their ids; a row's sum is the difference of two running sums
        order = torch.argsort(s["ids"], stable=True)
        first = torch.searchsorted(s["ids"][order], torch.arange(case["vocab"] + 1, dtype=torch.int32, device=DEV))
        out = torch.empty(case["vocab"], case["cols"], dtype=torch.float64, device=DEV)
        for a in range(0, case["cols"], 256):
            run_up = torch.nn.functional.pad(s["dy"][order, a:a + 256].double().cumsum(0), (0, 0, 1, 0))
            out[:, a:a + 256] = (run_up[first[1:]] - run_up[first[:-1]]) * s["scale"]
        return out
    if kind == "layernorm_grad":
        h, dy, gain = s["h"].double(), s["dy"].double(), s["gain"].double()
        xhat = (h - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        w = dy * gain
        inner = torch.einsum("td,td->t", w, xhat) / case["cols"]
        dx = s["dh"].double() + (w - w.sum(1, keepdim=True) / case["cols"] - xhat * inner[:, None]) * s["rstd"].double()[:, None]
        return {"dx": dx, "dgain": torch.einsum("td,td->d", dy, xhat), "dbias": torch.einsum("td->d", dy)}
    h = s["x"].double() + s["residual"].double()
    var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
    y = (h - mean) / torch.sqrt(var + EPS) * s["gain"].double() + s["bias"].double()
    if case["bits8"]:
        step = y.abs().max(dim=1, keepdim=True).values / 127.0
        y = torch.round(y / step) * step
    return {"h": h, "y": y}


# ------------------------------------------------------------------------------------------------- account
def work(case):
    kind, e = case["kind"], SIZE[case["type"]]
    if kind == "adamw":
        n = sum(sizes_of(case))
        kept = 2 * e if not case["master"] else 8 + e            # parameters read and written; with fp32 copies those are read
        moments = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
        return {"bytes": n * (e + kept + moments), "flops": 15.0 * n}
    T = case["tokens"]
    if kind == "score":
        V, k = case["vocab"], case["top"]
        return {"bytes": 1.0 * T * V * e + 8.0 * T * k + 16.0 * T, "flops": 6.0 * T * V}
    d = case["cols"]
    if kind == "embed":
        # a row that several tokens name is read once
        return {"bytes": (_distinct(0.9375 * T, case["vocab"]) + T) * d * e + 4.0 * T, "flops": 1.0 * T * d}
    if kind == "embed_grad":
        return {"bytes": 0.9375 * T * d * e + 1.0 * case["vocab"] * d * SIZE[case["out"]] + 4.0 * T, "flops": 1.0 * T * d}
    if kind == "layernorm":
        return {"bytes": T * d * (3.0 * e + (1.0 if case["bits8"] else e)) + 8.0 * d + (4.0 * T if case["bits8"] else 0.0),
                "flops": 8.0 * T * d}
    return {"bytes": 4.0 * T * d * e + 12.0 * d + 8.0 * T, "flops": 14.0 * T * d}


def _distinct(n, V):
    """Expected number of different ids among n tokens of _ids."""
    share = torch.log1p(1.0 / torch.arange(1, V + 1, dtype=torch.float64)) / math.log(V + 1.0)
    return float((1.0 - torch.exp(-n * share)).sum())
