"""The operators of language models around compressed layers, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` names what the user's program calls:

  product       x W^T with the weights held as 4-bit codes and a scale and an offset per group of columns
  product_grad  the gradient of its inputs, dy W: training around frozen codes
  norm          residual addition and root-mean-square norm, output in the inputs' type or in 8 bits
  norm_grad     its backward pass: gradients of the inputs and of the gain
  norm_product  a decoder layer's step into a 4-bit projection: residual addition, norm to 8 bits, product
  distill       loss of a student's logits against a teacher's top logits, with the student's gradient

`type` is that of activations, gradients and logits; scales, gains, losses and row weights are fp32.  Group 0
is one group for the whole row, the grid that the layer solver quantizes on.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # one token through the attention projection of a BERT-base sized transformer: latency is all it costs
        {"name": "product_1x768x768_bf16", "kind": "product", "tokens": 1, "rows": 768, "cols": 768, "group": 64,
         "type": "bf16"},
        # one token through a large square projection: the weights' bytes are all it costs
        {"name": "product_1x8192x8192_f16", "kind": "product", "tokens": 1, "rows": 8192, "cols": 8192, "group": 128,
         "type": "f16"},
        # a small decoding batch, nothing a multiple of a tile, rows of x not aligned to anything
        {"name": "product_13x5000x4999_bf16", "kind": "product", "tokens": 13, "rows": 5000, "cols": 4999, "group": 32,
         "type": "bf16"},
        # a prompt, or a training batch's forward pass, through a square projection
        {"name": "product_2048x4096x4096_bf16", "kind": "product", "tokens": 2048, "rows": 4096, "cols": 4096,
         "group": 128, "type": "bf16"},
        # a decoding step of eight sequences: residual, norm to 8 bits, feed-forward up-projection
        {"name": "norm_product_8x16384x4096_bf16", "kind": "norm_product", "tokens": 8, "rows": 16384, "cols": 4096,
         "group": 128, "type": "bf16"},
        # the same step for a prompt of a thousand tokens, finer groups
        {"name": "norm_product_1000x4096x8192_f16", "kind": "norm_product", "tokens": 1000, "rows": 4096, "cols": 8192,
         "group": 64, "type": "f16"},
        # backward pass of a training batch through a frozen square projection
        {"name": "product_grad_2048x4096x4096_bf16", "kind": "product_grad", "tokens": 2048, "rows": 4096,
         "cols": 4096, "group": 128, "type": "bf16"},
        # a small ragged fp32 batch through the layer solver's own grid, one scale a row
        {"name": "product_grad_77x2304x1283_f32", "kind": "product_grad", "tokens": 77, "rows": 2304, "cols": 1283,
         "group": 0, "type": "f32"},
        # norm of a training batch with its residual stream
        {"name": "norm_4096x8192_bf16", "kind": "norm", "tokens": 4096, "cols": 8192, "type": "bf16", "bits8": False},
        # and the backward pass of a narrower one
        {"name": "norm_grad_4096x4096_bf16", "kind": "norm_grad", "tokens": 4096, "cols": 4096, "type": "bf16"},
        # distillation of a short sequence on a small vocabulary
        {"name": "distill_48x32000_f16", "kind": "distill", "tokens": 48, "vocab": 32000, "top": 20, "type": "f16",
         "temperature": 1.0},
        # a training batch on a large one
        {"name": "distill_2048x131072_bf16", "kind": "distill", "tokens": 2048, "vocab": 131072, "top": 64,
         "type": "bf16", "temperature": 2.0},
    ]


# bounds on what draw() may give: half of the largest listed product, batch and set of logits
_MOST_MACS = 2 ** 34
_MOST_WEIGHTS = 2 ** 26
_MOST_ACTIVATIONS = 2 ** 24
_MOST_LOGITS = 2 ** 27


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["product", "product", "product", "norm_product", "product_grad", "norm", "norm_grad", "distill"])
    case = {"kind": kind, "type": rng.choice(["bf16", "f16", "f32"] if kind != "norm_product" else ["bf16", "f16"])}
    if kind in ("norm", "norm_grad"):
        case["cols"] = _log_int(rng, 64, 16384)
        case["tokens"] = _log_int(rng, 1, min(8192, _MOST_ACTIVATIONS // case["cols"]))
        if kind == "norm":
            case["bits8"] = rng.random() < 0.4
        return case
    if kind == "distill":
        case["vocab"] = _log_int(rng, 1000, 131072)
        case["tokens"] = _log_int(rng, 1, min(4096, _MOST_LOGITS // case["vocab"]))
        case["top"] = _log_int(rng, 1, 256)
        case["temperature"] = round(rng.uniform(0.5, 4.0), 2)
        return case
    case["rows"] = _log_int(rng, 64, 16384)
    case["cols"] = _log_int(rng, 64, min(16384, _MOST_WEIGHTS // case["rows"]))
    if rng.random() < 0.5:
        case["cols"] = (case["cols"] + 63) // 64 * 64
    case["tokens"] = _log_int(rng, 1, min(2048, _MOST_MACS // (case["rows"] * case["cols"])))
    case["group"] = rng.choice([32, 64, 128, 128, 256, 0])
    return case


# ------------------------------------------------------------------------------------------- inputs
def _tokens(T, d, gen):
    """Activations of a transformer: a few channels are ten times the others."""
    x = torch.randn(T, d, generator=gen, device=DEV)
    heavy = torch.randperm(d, generator=gen, device=DEV)[:max(1, round(0.01 * d))]
    x[:, heavy] *= 10.0
    return x


def _groups(case):
    """Columns of a group and groups of a row."""
    d = case["cols"]
    G = min(case["group"], d) if case["group"] else d
    return G, (d + G - 1) // G


def _weights(case, gen):
    """A layer rounded to its groups' min-max grids of 16 values: codes, steps and offsets (half-precision values)."""
    R, d = case["rows"], case["cols"]
    G, n = _groups(case)
    W = torch.randn(R, d, generator=gen, device=DEV) * 0.03
    pad = torch.nn.functional.pad(W, (0, n * G - d), value=float("nan")).view(R, n, G)
    lo = torch.where(pad.isnan(), float("inf"), pad).amin(2)
    hi = torch.where(pad.isnan(), float("-inf"), pad).amax(2)
    offset = lo.half().float()
    delta = torch.where(hi > lo, (hi - lo) / 15.0, 1.0).half().float()
    codes = torch.round((pad - offset[:, :, None]) / delta[:, :, None]).clamp(0, 15).nan_to_num(0.0)
    return codes.view(R, n * G)[:, :d].to(torch.int32), delta, offset


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kind, T, dt = case["kind"], case["tokens"], TYPES[case["type"]]
    s = {"case": case}
    if own:
        import paper_2208_11580_amd as obc
        s["ctx"] = obc.Context()
    if kind == "distill":
        V, k = case["vocab"], case["top"]
        z = torch.randn(T, V, generator=gen, device=DEV).mul_(3.0)
        s["z"] = z.to(dt)
        # the teacher agrees with the student in part; some of its rows list fewer than k tokens
        teacher = z.mul_(0.7).add_(torch.randn(T, V, generator=gen, device=DEV), alpha=2.0)
        top = teacher.topk(k, dim=1)
        s["top_logit"] = top.values.contiguous()
        count = torch.randint(max(1, k // 2), k + 1, (T, 1), generator=gen, device=DEV)
        s["top_index"] = torch.where(torch.arange(k, device=DEV) < count, top.indices, -1).to(torch.int32).contiguous()
        # an eighth of the tokens belong to the prompt and do not count
        s["weight"] = (torch.rand(T, generator=gen, device=DEV) < 0.875).float() / T
        if own:
            s["out"] = {"loss": torch.empty(T, device=DEV), "dz": torch.empty(T, V, dtype=dt, device=DEV)}
        return s
    d = case["cols"]
    if kind in ("product", "norm_product", "product_grad"):
        R = case["rows"]
        codes, s["delta"], s["offset"] = _weights(case, gen)
        if own:
            s["W"] = s["ctx"].obc_pack4(codes, s["delta"], s["offset"], group=case["group"])
            del s["delta"], s["offset"]
        else:
            # two codes to a byte
            pairs = torch.nn.functional.pad(codes, (0, d % 2)).view(R, -1, 2)
            s["W"] = (pairs[:, :, 0] + 16 * pairs[:, :, 1]).to(torch.uint8)
    if kind == "product":
        s["x"] = _tokens(T, d, gen).to(dt)
        if own:
            s["out"] = torch.empty(T, R, dtype=dt, device=DEV)
    elif kind == "product_grad":
        s["dy"] = (torch.randn(T, R, generator=gen, device=DEV) * 1e-3).to(dt)
        if own:
            s["out"] = torch.empty(T, d, dtype=dt, device=DEV)
    else:
        s["gain"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device=DEV)
        if kind == "norm_grad":
            h = _tokens(T, d, gen).to(dt)
            s["h"] = h
            s["rstd"] = (h.float().square().mean(1) + EPS).rsqrt()
            s["dy"] = (torch.randn(T, d, generator=gen, device=DEV) * 1e-3).to(dt)
            s["dh"] = (torch.randn(T, d, generator=gen, device=DEV) * 1e-3).to(dt)
            if own:
                s["out"] = {"dx": torch.empty(T, d, dtype=dt, device=DEV), "dgain": torch.empty(d, device=DEV)}
        else:
            s["x"] = _tokens(T, d, gen).mul_(0.3).to(dt)
            s["residual"] = _tokens(T, d, gen).to(dt)
            if own:
                s["out"] = {"h": torch.empty(T, d, dtype=dt, device=DEV)}
                if kind == "norm_product" or case["bits8"]:
                    s["out"]["y"] = torch.empty(T, d, dtype=torch.int8, device=DEV)
                    s["out"]["scale"] = torch.empty(T, device=DEV)
                else:
                    s["out"]["y"] = torch.empty(T, d, dtype=dt, device=DEV)
                if kind == "norm_product":
                    s["product"] = torch.empty(T, R, dtype=dt, device=DEV)
    return s


# --------------------------------------------------------------------------------- the framework's kernels
def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    kind = case["kind"]
    if kind == "product":
        return ctx.obc_product4(s["W"], s["x"], out=s["out"])
    if kind == "product_grad":
        return ctx.obc_product4_grad(s["W"], s["dy"], out=s["out"])
    if kind == "norm_grad":
        r = ctx.obc_rmsnorm_grad(s["h"], s["gain"], s["rstd"], s["dy"], dh=s["dh"], out=s["out"])
        return {"dx": r["dx"], "dgain": r["dgain"]}
    if kind == "distill":
        r = ctx.obc_distill(s["z"], s["top_index"], s["top_logit"], temperature=case["temperature"],
                            weight=s["weight"], want_grad=True, out=s["out"])
        return {"loss": r["loss"], "dz": r["dz"]}
    quant8 = kind == "norm_product" or case["bits8"]
    r = ctx.obc_rmsnorm(s["x"], s["gain"], eps=EPS, residual=s["residual"], quant8=quant8, out=s["out"])
    if kind == "norm_product":
        return {"h": r["h"], "y": ctx.obc_product4(s["W"], r["y"], x_scale=r["scale"], out=s["product"])}
    if quant8:
        return {"h": r["h"], "y": r["y"] * r["scale"][:, None]}      # the values that the 8 bits stand for
    return {"h": r["h"], "y": r["y"]}


# ------------------------------------------------------------------------------------------ the plain forms
def _dense(s):
    """The layer's weights in 32 bits from its bytes, steps and offsets."""
    case = s["case"]
    R, d = case["rows"], case["cols"]
    G, n = _groups(case)
    b = s["W"]
    codes = torch.stack((b & 15, b >> 4), dim=2).view(R, -1)[:, :d].float()
    if n == 1:
        return codes * s["delta"] + s["offset"]
    if n * G == d:
        return (codes.view(R, n, G) * s["delta"][:, :, None] + s["offset"][:, :, None]).view(R, d)
    g = torch.arange(d, device=DEV) // G
    return codes * s["delta"][:, g] + s["offset"][:, g]


def _norm(s):
    h = s["x"].float() + s["residual"].float()
    y = h * (h.square().mean(1, keepdim=True) + EPS).rsqrt() * s["gain"]
    return h, y


def _round8(y):
    """The values of y rounded to 8 bits with a scale for each row."""
    top = y.abs().amax(1, keepdim=True)
    scale = torch.where(top > 0, top / 127.0, 1.0)
    return torch.round(y / scale).clamp(-127, 127) * scale


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    kind, dt = case["kind"], TYPES[case["type"]]
    if kind == "product":
        return (s["x"].float() @ _dense(s).T).to(dt)
    if kind == "product_grad":
        return (s["dy"].float() @ _dense(s)).to(dt)
    if kind == "norm_grad":
        xhat = s["h"].float() * s["rstd"][:, None]
        dy = s["dy"].float()
        gy = dy * s["gain"]
        dx = s["dh"].float() + s["rstd"][:, None] * (gy - xhat * (gy * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(dt), "dgain": (dy * xhat).sum(0)}
    if kind == "distill":
        tau, idx = case["temperature"], s["top_index"]
        valid = idx >= 0
        t = torch.where(valid, s["top_logit"] / tau, float("-inf"))
        e = torch.exp(t - t.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
        logp = torch.where(valid, t - t.amax(1, keepdim=True) - e.sum(1, keepdim=True).log(), 0.0)
        z = s["z"].float() / tau
        top = z.amax(1, keepdim=True)
        lse = top + torch.exp(z - top).sum(1, keepdim=True).log()
        at = idx.clamp_min(0).long()
        logq = torch.gather(z, 1, at) - lse
        loss = s["weight"] * tau * tau * torch.where(valid, p * (logp - logq), 0.0).sum(1)
        dz = torch.exp(z - lse).scatter_add_(1, at, -p)
        return {"loss": loss, "dz": (dz * (tau * s["weight"])[:, None]).to(dt)}
    h, y = _norm(s)
    if kind == "norm_product":
        return {"h": h.to(dt), "y": (_round8(y) @ _dense(s).T).to(dt)}
    return {"h": h.to(dt), "y": _round8(y) if case["bits8"] else y.to(dt)}


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_product(x, codes, delta, offset, G):
    """Group by group: the codes' product times the step, and the inputs' sum times the offset."""
    y = torch.zeros(x.shape[0], codes.shape[0], dtype=torch.float64, device=DEV)
    for g in range(delta.shape[1]):
        xg, cg = x[:, g * G:(g + 1) * G], codes[:, g * G:(g + 1) * G].double()
        y += (xg @ cg.T) * delta[:, g].double()
        y += xg.sum(1, keepdim=True) * offset[:, g].double()
    return y


def exact(case, seed):
    global own
    kind, T = case["kind"], case["tokens"]
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if kind in ("product", "norm_product", "product_grad"):
        G, n = _groups(case)
        low, high = s["W"] % 16, s["W"] // 16
        codes = torch.empty(case["rows"], 2 * s["W"].shape[1], dtype=torch.uint8, device=DEV)
        codes[:, 0::2], codes[:, 1::2] = low, high
        codes = codes[:, :case["cols"]]
    if kind == "product":
        return _exact_product(s["x"].double(), codes, s["delta"], s["offset"], G)
    if kind == "product_grad":
        dy = s["dy"].double()
        parts = []
        for g in range(n):
            part = (dy * s["delta"][:, g].double()) @ codes[:, g * G:(g + 1) * G].double()
            parts.append(part + (dy @ s["offset"][:, g].double())[:, None])
        return torch.cat(parts, dim=1)
    if kind == "norm_grad":
        h, dy, r, gain = s["h"].double(), s["dy"].double(), s["rstd"].double(), s["gain"].double()
        dot = torch.einsum("td,td->t", dy * gain, h)
        dx = s["dh"].double() + (dy * gain) * r[:, None] - h * (dot * r ** 3 / case["cols"])[:, None]
        return {"dx": dx, "dgain": torch.einsum("td,td,t->d", dy, h, r)}
    if kind == "distill":
        tau = case["temperature"]
        loss = torch.zeros(T, dtype=torch.float64, device=DEV)
        dz = torch.empty(T, case["vocab"], dtype=torch.float64, device=DEV)
        for a in range(0, T, 256):
            z = s["z"][a:a + 256].double() / tau
            logq = torch.log_softmax(z, dim=1)
            valid = s["top_index"][a:a + 256] >= 0
            at = s["top_index"][a:a + 256].long() * valid
            logp = torch.log_softmax((s["top_logit"][a:a + 256].double() / tau).masked_fill(~valid, float("-inf")), dim=1)
            p = logp.exp()
            w = s["weight"][a:a + 256].double()
            terms = p * (logp.masked_fill(~valid, 0.0) - logq.gather(1, at))
            loss[a:a + 256] = w * tau ** 2 * terms.sum(1)
            full = torch.zeros_like(z).scatter_add_(1, at, p)
            dz[a:a + 256] = (logq.exp() - full) * (w * tau)[:, None]
        return {"loss": loss, "dz": dz}
    h = s["x"].double() + s["residual"].double()
    y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["cols"] + EPS) * s["gain"].double()
    if kind == "norm" and not case["bits8"]:
        return {"h": h, "y": y}
    step = y.abs().max(dim=1, keepdim=True).values / 127.0
    y8 = torch.round(y / step) * step
    if kind == "norm":
        return {"h": h, "y": y8}
    return {"h": h, "y": _exact_product(y8, codes, s["delta"], s["offset"], G)}


# ------------------------------------------------------------------------------------------------- account
def work(case):
    kind, T, e = case["kind"], case["tokens"], SIZE[case["type"]]
    if kind == "distill":
        V, k = case["vocab"], case["top"]
        return {"bytes": 2.0 * T * V * e + 8.0 * T * k + 8.0 * T, "flops": 8.0 * T * V}
    d = case["cols"]
    if kind == "norm":
        return {"bytes": T * d * (3.0 * e + (1.0 if case["bits8"] else e)) + 4.0 * d + (4.0 * T if case["bits8"] else 0.0),
                "flops": 5.0 * T * d}
    if kind == "norm_grad":
        return {"bytes": 4.0 * T * d * e + 8.0 * d + 4.0 * T, "flops": 10.0 * T * d}
    R = case["rows"]
    weights = 0.5 * R * d + 4.0 * R * _groups(case)[1]
    if kind == "norm_product":
        return {"bytes": weights + T * d * 3.0 * e + 4.0 * d + T * R * e, "flops": 2.0 * T * R * d + 5.0 * T * d}
    return {"bytes": weights + T * (d + R) * e, "flops": 2.0 * T * R * d}
